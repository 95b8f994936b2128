// The paged cache held in 4 bits: pages of the 16-bit cache are packed and read back, tokens are appended, and decode
// queries attend it, all of it or through a window with sinks.
//
// An element is e2m1 (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6); 32 channels of a token share
// a power of two 2^e, stored as the byte e + 127 (the OCP microscaling layout, whose conversions gfx950 has as
// instructions).  e is the smallest with max|x| <= 7 * 2^e, -126 at least: 7 rounds to 6, and is as far from it as any number
// is from its neighbours in the elements' last octave, so nothing loses more by saturation than by rounding.  A power of two
// for 32 channels and a rounding to the nearest element mean: an element is off by at most 2^e / 4 below 2 * 2^e, by 2^e / 2
// below 4 * 2^e and by 2^e above.  A block with an infinity or a NaN gets the byte 255 and reads as NaN.
// What is above 7/8 of a type's last power of two gets the element that stands for that power: 65536 for binary16 numbers above 57344 (an
// infinity when read back to binary16), 2^128 for bfloat16 ones above 1.75 * 2^127 (an infinity in any case).
//
// Record of one (page, KV head), 2176 bytes = 17 lines of 128:
//      0  keys' elements [token][channel / 2], even channel in the low half
//   1024  values' elements [token / 4][channel / 8][token % 4][channel % 8 / 2]
//   2048  keys' exponents [token][channel / 32]
//   2112  values' exponents [channel / 32][token]
// A wave's one 16-byte load per lane of the keys is then row lane % 16, channels 32 (lane / 16) .. + 31: the row operand of
// four matrix products (32 channels of one token share one power); its one load of the values is tokens 4 (lane / 16) .. + 3,
// channels 8 (lane % 16) .. + 7: what the lane gives to eight products whose weights it holds.
#include "psa_host.h"
#include "psa_visible.h"

namespace psa {

constexpr int kPackedBytes = PSA_PACKED_RECORD_BYTES;
constexpr int kPackedV = 1024, kPackedKExp = 2048, kPackedVExp = 2112;

// ---- elements -----------------------------------------------------------------------------------
// The power byte of a block from the bits (without sign) of its largest 16-bit value.
template <int DT>
__device__ __forceinline__ uint32_t power_byte(uint32_t top) {
    if (top >= (DT == 0 ? 0x7c00u : 0x7f80u)) return 255u;
    const uint32_t f = __float_as_uint(cvt_lo<DT>(top));
    // exponent of top, one more where its mantissa exceeds 1.75 = 7 / 4; minus 2 for 4 = 2^2
    const int e = (int)((f + 0x001fffffu) >> 23) - 2;
    return (uint32_t)max(e, 1);
}
// The scale operand of the conversions: a binary32 number whose exponent field is the byte (255 gives NaN).
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight 16-bit values (two a word) to eight elements, to nearest, ties to even, saturating.  NaN and infinity: zeros.
template <int DT>
__device__ __forceinline__ uint32_t to_elements(const uint4 &w, uint32_t byte) {
    const float s = power_of(byte);
    uint32_t c = 0;
    if constexpr (DT == 0) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, w.x), s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, w.y), s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, w.z), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, w.w), s, 3);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf2_t, w.x), s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf2_t, w.y), s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf2_t, w.z), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf2_t, w.w), s, 3);
    }
    return byte == 255u ? 0u : c;
}
// Eight elements to eight 16-bit values: exact in bfloat16 from 2^-126 to below 2^128, infinite in binary16 from 65536 on.
template <int DT>
__device__ __forceinline__ uint4 from_elements(uint32_t c, float s) {
    if constexpr (DT == 0) {
        return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 0)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 1)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 2)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 3)));
    } else {
        return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3)));
    }
}

// One row of 128 channels in sixteen lanes of eight: the lane's elements and its block's power byte.
template <int DT>
__device__ __forceinline__ uint32_t pack_row(const uint4 &w, uint32_t &byte) {
    uint32_t top = pk_max(pk_max(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), pk_max(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
    top = pk_max(top, dpp_u<0xB1>(top));                 // the four lanes of the block
    top = pk_max(top, dpp_u<0x4E>(top));
    byte = power_byte<DT>(max(top & 0xffffu, top >> 16));
    return to_elements<DT>(w, byte);
}

// Offset in a record of the value elements that a lane holds: token t, channels 8 cl .. 8 cl + 7.
__device__ __forceinline__ int value_offset(int t, int cl) { return kPackedV + ((t >> 2) * 64 + cl * 4 + (t & 3)) * 4; }

// ---- pages --------------------------------------------------------------------------------------
// Bound by memory: 8192 bytes in and 2176 out for a (listed page, KV head), one wave each; lane (rg, cl) takes rows 4 i + rg,
// channels 8 cl .. + 7, so loads are whole kilobytes and the stores of one instruction lie in 256 bytes.  8192 pages of 8 KV heads:
// 117 us = 5.8 TB/s, and 121 us back (a large copy: 4.9); 64 of them 3.5 us each way.
template <int DT>
__global__ __launch_bounds__(256) void pack_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                                                   uint8_t *__restrict__ packed, const int32_t *__restrict__ page_fill,
                                                   const int32_t *__restrict__ page_list, int num_units, int num_kv_heads,
                                                   int num_pages) {
    const int lane = threadIdx.x & 63, rg = lane >> 4, cl = lane & 15;
    const unsigned unit = blockIdx.x * 4u + (threadIdx.x >> 6);
    if (unit >= (unsigned)num_units) return;
    const int listed = unit / num_kv_heads, h = unit % num_kv_heads, page = page_list ? page_list[listed] : listed;
    if ((unsigned)page >= (unsigned)num_pages) return;   // a listed page outside the pool is skipped
    const int fill = page_fill ? min(max(page_fill[page], 0), kPage) : kPage;
    const size_t slice = (size_t)page * num_kv_heads + h;
    uint8_t *rec = packed + slice * kPackedBytes;
    Slice k = load_slice(k_pool + slice * kSliceBytes, lane), v = load_slice(v_pool + slice * kSliceBytes, lane);
    zero_invalid_rows(k, rg, fill);
    zero_invalid_rows(v, rg, fill);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 4 * i + rg;
        uint32_t kb, vb;
        *reinterpret_cast<uint32_t *>(rec + t * 64 + cl * 4) = pack_row<DT>(k.r[i], kb);
        *reinterpret_cast<uint32_t *>(rec + value_offset(t, cl)) = pack_row<DT>(v.r[i], vb);
        if ((cl & 3) == 0) {
            rec[kPackedKExp + t * 4 + (cl >> 2)] = (uint8_t)kb;
            rec[kPackedVExp + (cl >> 2) * 16 + t] = (uint8_t)vb;
        }
    }
}

template <int DT>
__global__ __launch_bounds__(256) void unpack_kernel(uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                                                     const uint8_t *__restrict__ packed, const int32_t *__restrict__ page_list,
                                                     int num_units, int num_kv_heads, int num_pages) {
    const int lane = threadIdx.x & 63, rg = lane >> 4, cl = lane & 15;
    const unsigned unit = blockIdx.x * 4u + (threadIdx.x >> 6);
    if (unit >= (unsigned)num_units) return;
    const int listed = unit / num_kv_heads, h = unit % num_kv_heads, page = page_list ? page_list[listed] : listed;
    if ((unsigned)page >= (unsigned)num_pages) return;
    const size_t slice = (size_t)page * num_kv_heads + h;
    const uint8_t *rec = packed + slice * kPackedBytes;
    uint8_t *ko = k_pool + slice * kSliceBytes + lane * 16, *vo = v_pool + slice * kSliceBytes + lane * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = 4 * i + rg;
        const uint32_t kc = *reinterpret_cast<const uint32_t *>(rec + t * 64 + cl * 4);
        const uint32_t vc = *reinterpret_cast<const uint32_t *>(rec + value_offset(t, cl));
        const float ks = power_of(rec[kPackedKExp + t * 4 + (cl >> 2)]), vs = power_of(rec[kPackedVExp + (cl >> 2) * 16 + t]);
        *reinterpret_cast<uint4 *>(ko + i * 1024) = from_elements<DT>(kc, ks);
        *reinterpret_cast<uint4 *>(vo + i * 1024) = from_elements<DT>(vc, vs);
    }
}

// One token per request: grid (batch), row group rg of wave w takes rows (key and value of KV heads) 4 w + rg, + 16, ...
template <int DT>
__global__ __launch_bounds__(256) void append_packed_kernel(uint8_t *__restrict__ packed, const int32_t *__restrict__ block_table,
                                                            int32_t *__restrict__ ctx_lens, const uint8_t *__restrict__ k_new,
                                                            const uint8_t *__restrict__ v_new, int32_t *__restrict__ status,
                                                            int num_kv_heads, int num_pages, int max_blocks) {
    const int r = blockIdx.x, cl = threadIdx.x & 15;
    const int ctx = ctx_lens[r];
    int err = 0, page = 0;
    if (ctx < 0 || ctx >= max_blocks * kPage) {
        err = PSA_DEVERR_CTX_RANGE;                 // no room in the request's row of the block table
    } else {
        page = block_table[(size_t)r * max_blocks + ctx / kPage];
        if ((unsigned)page >= (unsigned)num_pages) err = PSA_DEVERR_PAGE_RANGE;
    }
    if (!err) {
        const int t = ctx % kPage;
        for (int x = threadIdx.x >> 4; x < 2 * num_kv_heads; x += 16) {
            const int h = x >> 1, value = x & 1;
            const uint4 w = ld16((value ? v_new : k_new) + ((size_t)r * num_kv_heads + h) * kRowBytes + cl * 16);
            uint8_t *rec = packed + ((size_t)page * num_kv_heads + h) * kPackedBytes;
            uint32_t byte;
            const uint32_t c = pack_row<DT>(w, byte);
            *reinterpret_cast<uint32_t *>(rec + (value ? value_offset(t, cl) : t * 64 + cl * 4)) = c;
            if ((cl & 3) == 0) rec[value ? kPackedVExp + (cl >> 2) * 16 + t : kPackedKExp + t * 4 + (cl >> 2)] = (uint8_t)byte;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        if (!err) ctx_lens[r] = ctx + 1;
        if (status) status[r] = err;
    }
}

// ---- attention ----------------------------------------------------------------------------------
// What a lane holds of one page: 32 key elements of one token and their power, eight channels of four tokens' values
// and the four tokens' powers.
struct PackedPage {
    uint4 k, v;
    uint32_t kp, vp;
};
__device__ __forceinline__ PackedPage load_packed(const uint8_t *rec, uint32_t lane) {
    PackedPage p;
    const uint32_t rg = lane >> 4, cl = lane & 15;
    p.k = ld16_stream(rec + (cl * 64 + rg * 16));
    p.v = ld16_stream(rec + kPackedV + lane * 16u);
    p.kp = rec[kPackedKExp + (cl * 4 + rg)];
    p.vp = *reinterpret_cast<const uint32_t *>(rec + kPackedVExp + ((cl >> 2) * 16 + rg * 4));
    return p;
}
__device__ __forceinline__ uint32_t word_of(const uint4 &v, int w) { return w == 0 ? v.x : (w == 1 ? v.y : (w == 2 ? v.z : v.w)); }

// grid: one workgroup of four waves per piece (or request) and KV head, before them the one that checks the tables (if any).
// A wave takes pairs of visible blocks.
//   logits  D[token][row] = K[token][channel] Q[channel][row], four 16x16x32 products a block: elements and power become
//           bfloat16, exactly.  A query in bfloat16 stands in all rows of its head; one in binary16 is split into two
//           bfloat16 parts in neighbouring rows (8 + 3 bits, exact), whose sums are added.
//   values  D[row][channel] += P[row][token] V[token][channel], one 16x16x32 product for eight channels of the pair's 32
//           tokens.  Lane (rg, cl) has the logits of tokens 4 rg .. + 3 of both pages and loads just those tokens' values.
// (The matrix cores also take 4-bit elements and their powers as they are, with 8-bit floating parts of the query, but then
// add 128 products of different sizes with an error of 1e-5 of the sum of these sizes in the mean; these sums leave 1e-7.)
// Bound by memory: 4 requests of 128K tokens, 8 KV heads: 91 us = 6.3 TB/s at G = 4 (the call, with the launch that joins, 95),
// vector ALUs 46 % busy -- 64 conversions, 36 permutations and some 100 others for a pair of blocks --, matrix cores 12 %.  What brought
// it there from 173 us: the next pair under way (140), weight parts by masks and not by branches (127), table entries from
// a list that is loaded 64 blocks ahead and not each before its page (103).  Three pairs under way take as long; a workgroup needs
// two others on its CU (768 in all).
template <int DT, int G>
__global__ __launch_bounds__(256, 3) void packed_kernel(KvView kv, const uint8_t *__restrict__ q, VisiblePlan plan,
                                                        VisibleWs ws, float *__restrict__ out, float *__restrict__ lse) {
    constexpr int kRows = kRowsPerHead<G>;
    __shared__ __attribute__((aligned(16))) WaveSums<G> sums;
    const int tid = threadIdx.x, lane = tid & 63, rg = lane >> 4, cl = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);     // (so that table entries and page addresses are scalars)
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
    uint4 qb[4];                                         // B operand of the logits: channels 32 rg + 8 kk .. + 7
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        qb[kk] = make_uint4(0, 0, 0, 0);
        if (hd < G) qb[kk] = ld16(q + ((size_t)(r * kv.num_q_heads + h * G + hd) * kHeadDim + rg * 32 + kk * 8) * 2);
        if constexpr (DT == 0) {                         // binary16: the upper part in even rows, the rest in odd ones
            uint32_t w[4] = {qb[kk].x, qb[kk].y, qb[kk].z, qb[kk].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float a = cvt_lo<0>(w[j]), b = cvt_hi<0>(w[j]);
                if (part & 1) {
                    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                    b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
                }
                w[j] = (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xffff0000u);
            }
            qb[kk] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    float ref = 0.0f, limit = -INFINITY, l = 0.0f;       // head hd: see raise_reference; exp-sum of this row group
    f32x4_t acc[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    const int32_t *table = kv.block_table + (size_t)r * kv.max_blocks;
    // Lane j holds the page of the j-th block of the wave's next 64 (32 pairs); the list after it is under way.
    auto list_of = [&](int b) __attribute__((always_inline)) { return table[vis.block(min(b + 8 * (lane >> 1) + (lane & 1), b1 - 1))]; };
    int pages = 0, later = 0;
    auto load_pair = [&](PackedPage (&x)[2], int b, int i) __attribute__((always_inline)) {      // the wave's i-th pair
        if ((i & 31) == 0) {
            const int page = i == 0 ? list_of(b) : later;
            pages = clamp_page_quiet(page, kv.num_pages);
            if (pages != page) err |= PSA_DEVERR_PAGE_RANGE;
            later = list_of(b + 256);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y)
            x[y] = load_packed(kv.k_pool + ((size_t)__builtin_amdgcn_readlane(pages, 2 * (i & 31) + y) * kv.num_kv_heads + h) * kPackedBytes, lane);
    };
    auto attend_pair = [&](PackedPage (&pg)[2], int b) __attribute__((always_inline)) {
        float sc[8];                                     // (not yet scaled)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            f32x4_t d = {0.0f, 0.0f, 0.0f, 0.0f};
            const float ks = power_of(pg[y].kp);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) d = mfma_16x16x32<1>(from_elements<1>(word_of(pg[y].k, kk), ks), qb[kk], d);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sc[4 * y + j] = d[j];
                if constexpr (DT == 0) sc[4 * y + j] += dpp_f<0xB1>(sc[4 * y + j]);
            }
            const int lb = vis.block(b + y);
            if (b + y >= b1 || !vis.sees_all(lb)) {
                uint32_t vw[4] = {pg[y].v.x, pg[y].v.y, pg[y].v.z, pg[y].v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool seen = (b + y < b1) & vis.sees(lb * kPage + 4 * rg + j);
                    sc[4 * y + j] = seen ? sc[4 * y + j] : -INFINITY;
                    vw[j] = seen ? vw[j] : 0u;           // (the power may be NaN: its byte goes as well)
                    pg[y].vp &= seen ? ~0u : ~(0xffu << (8 * j));
                }
                pg[y].v = make_uint4(vw[0], vw[1], vw[2], vw[3]);
            }
        }
        const float bm = kScaleLog2 * fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
        if (__ballot(bm > limit)) raise_reference(bm, ref, limit, l, acc, rg);
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = exp2_fast(fmaf(sc[j], kScaleLog2, -ref));
        l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        uint4 a[kProducts<G>];
#pragma unroll
        for (int y = 0; y < kProducts<G>; ++y)
            a[y] = make_uint4(parts(p[0], p[1], y), parts(p[2], p[3], y), parts(p[4], p[5], y), parts(p[6], p[7], y));
        float power[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) power[j] = power_of((pg[j >> 2].vp >> (8 * (j & 3))) & 0xffu);
        static_for<4>([&](auto u) __attribute__((always_inline)) {      // channels 2 u and 2 u + 1 of the lane's eight
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word_of(pg[j >> 2].v, j & 3), power[j], u));
            const uint4 even = make_uint4(pick_halves<false>(x[0], x[1]), pick_halves<false>(x[2], x[3]),
                                          pick_halves<false>(x[4], x[5]), pick_halves<false>(x[6], x[7]));
            const uint4 odd = make_uint4(pick_halves<true>(x[0], x[1]), pick_halves<true>(x[2], x[3]),
                                         pick_halves<true>(x[4], x[5]), pick_halves<true>(x[6], x[7]));
#pragma unroll
            for (int y = 0; y < kProducts<G>; ++y) {
                acc[2 * u] = mfma_16x16x32<1>(a[y], even, acc[2 * u]);
                acc[2 * u + 1] = mfma_16x16x32<1>(a[y], odd, acc[2 * u + 1]);
            }
        });
    };
    // The next pair is under way while one is worked on, in two sets of registers that take turns.  Loads beyond the last block
    // read that one again, so that no branch hides from the compiler how many are outstanding.
    PackedPage x0[2], x1[2];
    const int first = b0 + 2 * wave;
    if (first < b1) {
        load_pair(x0, first, 0);
        for (int b = first, i = 0; b < b1; b += 16, i += 2) {
            load_pair(x1, b + 8, i + 1);
            attend_pair(x0, b);
            if (b + 8 >= b1) break;
            load_pair(x0, b + 16, i + 2);
            attend_pair(x1, b + 8);
        }
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

// ---- host side ----------------------------------------------------------------------------------
hipError_t launch_pack(const psa_kv_desc *d, void *packed, const int32_t *page_fill, const int32_t *page_list, int num_listed,
                       hipStream_t st) {
    const long long units = (long long)(page_list ? num_listed : d->num_pages) * d->num_kv_heads;
    if (units == 0) return hipSuccess;
    const unsigned grid = (unsigned)((units + 3) / 4);
    (d->dtype == PSA_F16 ? pack_kernel<0> : pack_kernel<1>)<<<grid, 256, 0, st>>>(
        (const uint8_t *)d->k_pool, (const uint8_t *)d->v_pool, (uint8_t *)packed, page_fill, page_list, (int)units, d->num_kv_heads,
        d->num_pages);
    return hipGetLastError();
}

hipError_t launch_unpack(const psa_kv_desc *d, const void *packed, const int32_t *page_list, int num_listed, hipStream_t st) {
    const long long units = (long long)(page_list ? num_listed : d->num_pages) * d->num_kv_heads;
    if (units == 0) return hipSuccess;
    const unsigned grid = (unsigned)((units + 3) / 4);
    (d->dtype == PSA_F16 ? unpack_kernel<0> : unpack_kernel<1>)<<<grid, 256, 0, st>>>(
        (uint8_t *)d->k_pool, (uint8_t *)d->v_pool, (const uint8_t *)packed, page_list, (int)units, d->num_kv_heads, d->num_pages);
    return hipGetLastError();
}

hipError_t launch_append_packed(const psa_kv_desc *d, void *packed, const void *k_new, const void *v_new, int32_t *status,
                                hipStream_t st) {
    (d->dtype == PSA_F16 ? append_packed_kernel<0> : append_packed_kernel<1>)<<<d->batch, 256, 0, st>>>(
        (uint8_t *)packed, d->block_table, (int32_t *)d->ctx_lens, (const uint8_t *)k_new, (const uint8_t *)v_new, status,
        d->num_kv_heads, d->num_pages, d->max_blocks_per_seq);
    return hipGetLastError();
}

// 768 workgroups: see the kernel.  Pieces of 32 blocks at least: one request of 32K tokens takes 14.4 us, 16.5 with 16, 16.2 with 48.  One
// launch up to 320 blocks from 192 (request, KV head) pairs on: 64 requests of 8 KV heads with windows of 2040 tokens 28 us (39 in
// pieces), of 4000 49 (57), of 8000 77 (69); 32 requests of 1024 tokens 11.4 (14.9), of 4096 30.7 (33.4); 16 requests of 1024 9.6 (11.9),
// of 2048 15.4 (15.3), of 4096 26.8 (22.3).
constexpr int kPackedGroups = 768, kPackedLeastBlocks = 32, kPackedDirectFrom = 192;
static VisiblePlan packed_plan(const psa_kv_desc *d, int window, int num_sinks) {
    return visible_plan(d, window, num_sinks, kPackedGroups, kPackedLeastBlocks, kPackedDirectFrom);
}

size_t packed_workspace_bytes(const psa_kv_desc *d, int window, int num_sinks) {
    return visible_workspace_bytes(d, packed_plan(d, window, num_sinks));
}

template <int DT, int G>
static hipError_t launch_packed_t(const KvView &kv, const void *q, const VisiblePlan &plan, const VisibleWs &ws, float *out, float *lse,
                                  hipStream_t st) {
    const unsigned grid = (unsigned)(kv.num_kv_heads * (plan.direct ? kv.batch : plan.groups + kv.batch) + plan.checked);
    if (plan.direct && !plan.checked && launch_clear(ws.header, st) != hipSuccess) return hipErrorLaunchFailure;
    if (plan.listed && launch_list(kv, plan, ws, st) != hipSuccess) return hipErrorLaunchFailure;
    packed_kernel<DT, G><<<grid, 256, 0, st>>>(kv, (const uint8_t *)q, plan, ws, out, lse);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && !plan.direct ? launch_join(kv, plan, ws, out, lse, st) : e;
}

hipError_t launch_packed(const psa_kv_desc *d, const void *packed, const void *q, int window, int num_sinks, float *out, float *lse,
                         void *ws, hipStream_t st) {
    KvView kv = make_view(d);
    kv.k_pool = static_cast<const uint8_t *>(packed);
    kv.v_pool = nullptr;
    if (kv.num_pages == 0) {
        DecodeArgs a{};
        a.out = out;
        a.lse_out = lse;
        return launch_no_pages(kv, a, reinterpret_cast<int32_t *>(ws), st);
    }
    const int G = d->num_q_heads / d->num_kv_heads;
    const VisiblePlan plan = packed_plan(d, window, num_sinks);
    const VisibleWs vws = visible_ws(d, plan, ws);
#define PSA_CASE(DT, GG) \
    if (d->dtype == DT && G == GG) return launch_packed_t<DT, GG>(kv, q, plan, vws, out, lse, st);
    PSA_CASE(0, 1) PSA_CASE(0, 2) PSA_CASE(0, 4) PSA_CASE(0, 8)
    PSA_CASE(1, 1) PSA_CASE(1, 2) PSA_CASE(1, 4) PSA_CASE(1, 8)
#undef PSA_CASE
    return hipErrorInvalidValue;
}

}  // namespace psa
