// Queries and keys made ready for the cache in one pass: RMS norm of every head, then the rotation of its first rot_dim
// channels by the token's position.
//   y = x / sqrt(mean(x^2) + eps) * w            (if normalised; w = 1 without weights)
//   pair i of frequency f_i: (a, b) -> (a cos - b sin, a sin + b cos), angle = position * f_i
// Everything in binary32, rounded once to the type of x; the angle is formed and reduced to a fraction of a turn in binary64
// (position * f_i has up to 55 bits; at position 2^20 binary32 would leave an error of 0.03 radians), its sine and cosine in binary32.
//
// Sixteen lanes hold a head's row; a lane's eight channels are four pairs, always of the frequencies 4 cl .. 4 cl + 3, so a
// lane finds four sines and cosines once per token and uses them for all heads that its wave takes: no table, no exchange.
// Pairs (i, i + rot_dim / 2) are two loads of four channels, pairs (2 i, 2 i + 1) one load of eight; what lies beyond
// rot_dim fills the remaining places and passes through.
// Bound by memory for prompts (256 bytes in and out for a row): 16384 tokens of 32 + 8 heads 69 us = 4.9 TB/s, a large copy's rate
// (75 us without the streaming hints and one row at a time).  One token 3.1 us, of which the launch is most: its ten waves take four
// rows each (7.0 us with one wave for all forty, one after the other).  Between them a wave waits for the position, then for four
// sines and cosines, then for its rows: 1024 tokens of 32 + 8 heads 9.4 us = 2.2 TB/s, 4096 23.4 us = 3.6.
#include "psa_attend.h"
#include "psa_host.h"

namespace psa {

struct RotateArgs {
    const uint8_t *q_in, *k_in;
    uint8_t *q_out, *k_out;
    const uint8_t *q_weight, *k_weight;
    const int32_t *positions;
    const float *inv_freq;
    long long q_in_stride, k_in_stride, q_out_stride, k_out_stride;   // bytes from token to token
    int tokens, q_heads, kv_heads, half, normalize, rows_per_wave, waves_per_token;
    float eps;
};

typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ void widen(const u32x2_t &w, float *x) {
    x[0] = cvt_lo<DT>(w.x); x[1] = cvt_hi<DT>(w.x); x[2] = cvt_lo<DT>(w.y); x[3] = cvt_hi<DT>(w.y);
}
template <int DT>
__device__ __forceinline__ uint32_t round16(float a, float b) {
    if constexpr (DT == 0) {
        const half2_t h = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, h);
    } else {
        const bf2_t h = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, h);
    }
}

// One wave: rows_per_wave rows (heads, queries first) of one token, four at a time.
// PAIRED: pairs (2 i, 2 i + 1); otherwise (i, i + half).
template <int DT, bool PAIRED>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a) {
    const int lane = threadIdx.x & 63, rg = lane >> 4, cl = lane & 15;
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long token = wave / a.waves_per_token;
    if (token >= a.tokens) return;
    const int first = (int)(wave % a.waves_per_token) * a.rows_per_wave;
    const int rows = a.q_heads + a.kv_heads, last = min(rows, first + a.rows_per_wave);
    float c[4], s[4];
    // first channels of the lane's two groups of four (PAIRED: eight neighbours, pairs interleaved)
    const int i0 = 4 * cl, lo = PAIRED ? 8 * cl : (i0 < a.half ? i0 : a.half + i0), hi = PAIRED ? 8 * cl + 4 : (i0 < a.half ? i0 + a.half : 64 + i0);
    const double position = a.half ? (double)a.positions[token] : 0.0;      // (without rotation there may be none)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c[j] = 1.0f;
        s[j] = 0.0f;
        if (i0 + j < a.half) {
            const double turns = position * (double)a.inv_freq[i0 + j] * 0.15915494309189533576888;     // 1 / (2 pi)
            const float t = (float)(turns - rint(turns));                                             // -1/2 .. 1/2 of a turn
            sincospif(2.0f * t, &s[j], &c[j]);
        }
    }
    // what streams through is marked read (written) once
    auto load = [&](int row, float (&x)[8]) __attribute__((always_inline)) {
        const uint8_t *src = row < a.q_heads ? a.q_in + token * a.q_in_stride + row * kRowBytes
                                             : a.k_in + token * a.k_in_stride + (row - a.q_heads) * kRowBytes;
        widen<DT>(__builtin_nontemporal_load(reinterpret_cast<const u32x2_t *>(src + 2 * lo)), x);
        widen<DT>(__builtin_nontemporal_load(reinterpret_cast<const u32x2_t *>(src + 2 * hi)), x + 4);
    };
    auto finish = [&](int row, float (&x)[8]) __attribute__((always_inline)) {
        const bool is_q = row < a.q_heads;
        if (a.normalize) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
            sum = row_sum16(sum);
            float eps = a.eps;
            // Squares beyond binary32 (bfloat16 numbers above 2^60; below 2^-50 if eps is as good as none): the row and eps are
            // scaled by a power of two first, which the quotient does not see.  All lanes of a row go the same way.
            if (!(sum < INFINITY) || sum + kHeadDim * eps < 0x1p-90f) {
                const float scale = sum > 1.0f ? 0x1p-80f : 0x1p80f;
                sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] *= scale;
                    sum = fmaf(x[j], x[j], sum);
                }
                sum = row_sum16(sum);
                eps = eps * scale * scale;
            }
            const float f = 1.0f / sqrtf(sum * (1.0f / kHeadDim) + eps);
            const uint8_t *w = is_q ? a.q_weight : a.k_weight;
            float g[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
            if (w) {
                widen<DT>(*reinterpret_cast<const u32x2_t *>(w + 2 * lo), g);
                widen<DT>(*reinterpret_cast<const u32x2_t *>(w + 2 * hi), g + 4);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = x[j] * f * g[j];
        }
        float y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int u = PAIRED ? 2 * j : j, v = PAIRED ? 2 * j + 1 : j + 4;
            const bool turned = i0 + j < a.half;         // (what passes through is no sum: it may be infinite)
            y[u] = turned ? x[u] * c[j] - x[v] * s[j] : x[u];
            y[v] = turned ? x[u] * s[j] + x[v] * c[j] : x[v];
        }
        uint8_t *dst = is_q ? a.q_out + token * a.q_out_stride + row * kRowBytes
                            : a.k_out + token * a.k_out_stride + (row - a.q_heads) * kRowBytes;
        __builtin_nontemporal_store(u32x2_t{round16<DT>(y[0], y[1]), round16<DT>(y[2], y[3])}, reinterpret_cast<u32x2_t *>(dst + 2 * lo));
        __builtin_nontemporal_store(u32x2_t{round16<DT>(y[4], y[5]), round16<DT>(y[6], y[7])}, reinterpret_cast<u32x2_t *>(dst + 2 * hi));
    };
    for (int row = first + rg; row < last; row += 8) {   // two rows' loads before either's stores: both may be in place
        float x[2][8];
        const bool second = row + 4 < last;
        load(row, x[0]);
        if (second) load(row + 4, x[1]);
        finish(row, x[0]);
        if (second) finish(row + 4, x[1]);
    }
}

// Below this many tokens a token's rows are spread over several waves, up to this many waves in all (bfloat16; with four times as many
// waves, and with a quarter of them): 512 tokens of 32 + 8 heads 5.2 us (5.7, 6.1), 1024 9.4 (11.0, 13.1), 2048 13.9 (15.0, 17.0), 4096 23.4
// (24.5, 23.5), 8192 36.4 (38.2, 35.9); 1024 tokens of 8 + 1 heads 4.8 (4.7, 5.7), 4096 9.4 (11.5, 9.4).
constexpr int kRotateWaves = 4096;

hipError_t launch_rotate(const psa_rotate_desc *d, const void *q_in, const void *k_in, void *q_out, void *k_out, const void *q_weight,
                         const void *k_weight, const int32_t *positions, const float *inv_freq, hipStream_t st) {
    RotateArgs a;
    a.q_in = (const uint8_t *)q_in;
    a.k_in = (const uint8_t *)k_in;
    a.q_out = (uint8_t *)q_out;
    a.k_out = (uint8_t *)k_out;
    a.q_weight = (const uint8_t *)q_weight;
    a.k_weight = (const uint8_t *)k_weight;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.q_in_stride = 2 * d->q_in_stride;
    a.k_in_stride = 2 * d->k_in_stride;
    a.q_out_stride = 2 * d->q_out_stride;
    a.k_out_stride = 2 * d->k_out_stride;
    a.tokens = d->num_tokens;
    a.q_heads = d->num_q_heads;
    a.kv_heads = d->num_kv_heads;
    a.half = d->rot_dim / 2;
    a.normalize = d->normalize;
    a.eps = d->eps;
    // a wave takes all rows of its token where there are tokens enough to fill the GPU; fewer, down to four, where there are not
    const int quads = (a.q_heads + a.kv_heads + 3) / 4;
    const int want = a.tokens >= kRotateWaves ? 1 : (kRotateWaves + a.tokens - 1) / a.tokens, most = want < quads ? want : quads;
    const int per_wave = (quads + most - 1) / most;
    a.rows_per_wave = 4 * per_wave;
    a.waves_per_token = (quads + per_wave - 1) / per_wave;
    const long long waves = (long long)a.tokens * a.waves_per_token;
    const unsigned grid = (unsigned)((waves + 3) / 4);
    auto kernel = d->dtype == PSA_F16 ? (d->interleaved ? rotate_kernel<0, true> : rotate_kernel<0, false>)
                                      : (d->interleaved ? rotate_kernel<1, true> : rotate_kernel<1, false>);
    kernel<<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace psa
