// Norm of queries and keys per head and their rotation by position, forward and backward; the same on the way into a paged cache.
//
//   z = x r w,  r = (mean of the head's x^2 + eps)^-1/2      (without a weight: z = x)
//   (y_a, y_b) = (z_a cos - z_b sin, z_a sin + z_b cos)      for the pairs (a, b) of the first `rot` values, angle = position * frequency
//   backward: dz = dy turned back;  dw = sum of dz x r over tokens and heads;  dx = r (w dz - x r * mean(w dz x r))
//
// A head is at most 32 chunks of eight values.  G lanes share it, two chunks each: the chunks of a pair's two halves, so that a pair never
// leaves its lane, and the rest beside each other.  Angles are the same for every head of a token: a wave works each out once, a lane a pair, and
// hands them round through shared memory.  Everything between the 16-bit input and the 16-bit output is 32 bits, angles 64.
#pragma once

#include <cmath>
#include <type_traits>

#include "launch.h"
#include "mfma.h"
#include "sequences.h"

namespace mmee {

struct Rows {                   // a tensor's strides in elements
    int64_t token, head;
};

struct RotateArgs {
    uint32_t tokens, heads, kv_heads, head_dim, rot;
    uint32_t axes, shares;      // shares: waves that share a token's heads
    float eps;
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out, *v_out;            // k_out, v_out: tensors, or pages
    Rows qs, ks, vs, qos, kos, vos;
    const uint16_t *q_weight, *k_weight;
    const double *freqs;
    const int32_t *positions;
    int64_t axis_stride;
    const uint8_t *axis_of;
    // paged cache
    int64_t k_page, v_page, table_stride;       // from one page, and from one sequence's entries, to the next
    const int32_t *starts, *counts, *cache_lens, *page_table;
    uint32_t seqs, per_seq, page_shift, pages_per_seq, n_pages;
    // backward
    const uint16_t *dq_out, *dk_out;
    uint16_t *dq, *dk, *dq_weight, *dk_weight;
    Rows dqos, dkos, dqs, dks;
    float *parts;               // [block][2][head_dim]
    uint32_t blocks;
};

// cos and sin of position * frequency.  The product in turns in 64 bits, which a million turns away still tell 2^-33 of a turn apart; the
// eighth of a turn that is left, in 32 bits, by the Taylor series, whose next terms are below 2^-28.
__device__ __forceinline__ void turn(double position, double freq, float &cos, float &sin)
{
    constexpr double PER_TURN = 0.15915494309189533577;
    const double turns = position * (freq * PER_TURN);
    const float part = (float)(turns - __builtin_rint(turns));              // -1/2 .. 1/2
    const float quarters = __builtin_rintf(4.0f * part);
    const float x = (part - 0.25f * quarters) * 6.2831853071795865f, x2 = x * x;            // |x| <= pi / 4
    const float s = x + x * x2 * (-1.0f / 6 + x2 * (1.0f / 120 + x2 * (-1.0f / 5040 + x2 * (1.0f / 362880))));
    const float c = 1.0f + x2 * (-0.5f + x2 * (1.0f / 24 + x2 * (-1.0f / 720 + x2 * (1.0f / 40320 - x2 * (1.0f / 3628800)))));
    const int n = (int)quarters & 3;
    const float a = n & 1 ? s : c, b = n & 1 ? c : s;
    cos = n == 1 || n == 2 ? -a : a;
    sin = n & 2 ? -b : b;
}

// What a lane holds of a head: chunks at[0] and at[1] (of eight values), values a[0..7], b[0..7].
template <class T, int G, bool NEIGHBOURS>
struct Head {
    uint32_t at[2];
    bool there[2], turned[2];
    float cos[8], sin[8];       // halves: of the pairs (a[j], b[j]); neighbours: 0..3 of a's pairs, 4..7 of b's

    __device__ __forceinline__ explicit Head(const RotateArgs &r)
    {
        const uint32_t p = threadIdx.x % G, chunks = r.head_dim / 8, half = NEIGHBOURS ? 0 : r.rot / 16, lanes = (chunks + 1) / 2;
        at[0] = p < half ? p : half + p;                                    // (2 half + p - half)
        at[1] = p < half ? p + half : at[0] + (lanes - half);
        there[0] = p < lanes;
        there[1] = p < lanes && at[1] < chunks;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            turned[i] = there[i] && 8 * at[i] < r.rot;
            if (!there[i]) at[i] = 0;
        }
    }

    // shared: this wave's, cosines and sines of the pairs.  (Worked out by every lane that needs them it took a third of the time of 12000 tokens of 24 heads of 64.)
    __device__ __forceinline__ void angles(const RotateArgs &r, uint32_t token, int64_t place, float (&shared)[2][128])
    {
        wave_sync();                                    // of the token before
        for (uint32_t pair = threadIdx.x & 63; 2 * pair < r.rot; pair += 64) {
            double position = (double)place;
            if (r.positions) {
                const uint32_t axis = r.axis_of ? r.axis_of[pair] : 0;
                position = r.positions[(axis < r.axes ? axis : r.axes - 1) * r.axis_stride + token];
            }
            turn(position, r.freqs[pair], shared[0][pair], shared[1][pair]);
        }
        wave_sync();
    }

    // This lane's.
    __device__ __forceinline__ void take(const float (&shared)[2][128])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t first = NEIGHBOURS ? 4 * at[i] : 8 * at[0] + 4 * i;
            const f32x4 c = *reinterpret_cast<const f32x4 *>(&shared[0][first & 127]), s = *reinterpret_cast<const f32x4 *>(&shared[1][first & 127]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                cos[4 * i + j] = c[j];
                sin[4 * i + j] = s[j];
            }
        }
    }

    __device__ __forceinline__ void load(const uint16_t *head, u32x4 (&raw)[2]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            raw[i] = u32x4{0, 0, 0, 0};
            if (there[i]) raw[i] = *reinterpret_cast<const u32x4 *>(head + 8 * at[i]);
        }
    }

    static __device__ __forceinline__ void widen(const u32x4 (&raw)[2], float (&x)[16])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x8 y = __builtin_convertvector(as_operand<T>(raw[i]), f32x8);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[8 * i + j] = y[j];
        }
    }

    __device__ __forceinline__ void store(uint16_t *head, const float (&x)[16]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x8 y;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = x[8 * i + j];
            if (there[i]) *reinterpret_cast<typename T::V8 *>(head + 8 * at[i]) = __builtin_convertvector(y, typename T::V8);
        }
    }

    // sign = 1: by the angles; -1: back.
    __device__ __forceinline__ void rotate(float (&x)[16], float sign) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int a = NEIGHBOURS ? 8 * (j / 4) + 2 * (j % 4) : j, b = NEIGHBOURS ? a + 1 : 8 + j;
            const float s = sign * sin[j], u = x[a] * cos[j] - x[b] * s, w = x[a] * s + x[b] * cos[j];
            const bool yes = turned[NEIGHBOURS ? j / 4 : 0];
            x[a] = yes ? u : x[a];
            x[b] = yes ? w : x[b];
        }
    }

    // Of the head's G lanes, 1, 2, 4 and 8 apart.
    static __device__ __forceinline__ float sum(float x)
    {
        const auto add = [&x](auto apart) { x += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), apart.value << 10 | 0x1f)); };
        add(std::integral_constant<int, 1>());
        if constexpr (G > 2) add(std::integral_constant<int, 2>());
        if constexpr (G > 4) add(std::integral_constant<int, 4>());
        if constexpr (G > 8) add(std::integral_constant<int, 8>());
        return x;
    }

    static __device__ __forceinline__ float squares(const float (&x)[16])
    {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) s += x[j] * x[j];
        return sum(s);
    }

    // (mean of the head's x^2 + eps)^-1/2.  Where the squares pass 32 bits, in bfloat16 from 2^60 on, those of 2^-96 times the head are summed, next to which eps is nothing.
    static __device__ __forceinline__ float inverse_root(const float (&x)[16], const RotateArgs &r)
    {
        const float s = squares(x);
        float inverse = __builtin_amdgcn_rsqf(s / (float)r.head_dim + r.eps);
        if (std::is_same<T, BF16>::value && __any(s == INFINITY)) {
            float t = 0.0f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float y = 0x1p-96f * x[j];
                t += y * y;
            }
            t = sum(t);
            if (s == INFINITY) inverse = 0x1p-96f * __builtin_amdgcn_rsqf(t / (float)r.head_dim);
        }
        return inverse;
    }
};

// Forward: a wave takes 64 / G heads of a token at a time.  CACHE: keys and values go to the pages, values as they are.
// Bound by HBM where there are many tokens, each value read and written once: 16384 tokens of 32 and 8 heads of 128, 336 MB, 63 us, 5.3 TB/s; 17989 tokens on
// their way to pages of 64, 442 MB, 90 us, 4.9 TB/s; heads of 80, neighbours paired, 84 MB, 17 us, 4.8 TB/s.  One token: 2.8 us, 64 sequences' next
// ones 4.0: a launch, and the trips for the page or the position, its angle and the head, one after the other.
template <class T, int G, bool NEIGHBOURS, bool CACHE>
__global__ __launch_bounds__(256) void k_rotate(const RotateArgs r)
{
    constexpr uint32_t PER = 64 / G;
    __shared__ __align__(16) float shared[4][2][128];
    const uint64_t wave = (uint64_t)blockIdx.x * (blockDim.x / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t token = (uint32_t)(wave / r.shares), share = (uint32_t)(wave % r.shares);
    if (token >= r.tokens) return;
    int64_t place = 0;
    int32_t page = -1;
    if (CACHE) {
        int seq = r.starts ? last_at_most(r.seqs, token, [&](uint32_t i) { return (int64_t)r.starts[i]; }) : (int)(token / r.per_seq);
        seq = __builtin_amdgcn_readfirstlane(seq);
        if (seq < 0 || (r.starts && (int64_t)token >= r.starts[seq + 1])) return;           // a token of no sequence
        const int64_t nth = r.starts ? (int64_t)token - r.starts[seq] : token % r.per_seq;
        if (r.counts && nth >= r.counts[seq]) return;
        place = within(r.cache_lens[seq], 0, INT32_MAX) + nth;
        if (place >> r.page_shift < r.pages_per_seq) page = r.page_table[seq * r.table_stride + (place >> r.page_shift)];
        if ((uint32_t)page >= r.n_pages) page = -1;
    }
    Head<T, G, NEIGHBOURS> h(r);
    const uint32_t own_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    h.angles(r, token, place, shared[own_wave]);
    h.take(shared[own_wave]);
    float w[2][16];
    const bool norm = r.q_weight || r.k_weight;
    if (norm) {
        u32x4 raw[2];
        h.load(r.q_weight, raw);
        h.widen(raw, w[0]);
        h.load(r.k_weight, raw);
        h.widen(raw, w[1]);
    }
    const uint32_t all = r.heads + r.kv_heads * (CACHE ? 2 : 1);
    const int64_t inside = CACHE ? place & ((1u << r.page_shift) - 1) : 0;
    for (uint32_t at = share * PER + (threadIdx.x & 63) / G; at - (threadIdx.x & 63) / G < all; at += r.shares * PER) {
        if (at >= all) continue;
        const bool is_q = at < r.heads, is_v = CACHE && at >= r.heads + r.kv_heads;
        const uint32_t head = is_q ? at : is_v ? at - r.heads - r.kv_heads : at - r.heads;
        const uint16_t *from = is_q ? r.q + token * r.qs.token + head * r.qs.head : is_v ? r.v + token * r.vs.token + head * r.vs.head : r.k + token * r.ks.token + head * r.ks.head;
        uint16_t *to;
        if (is_q) to = r.q_out + token * r.qos.token + head * r.qos.head;
        else if (!CACHE) to = r.k_out + token * r.kos.token + head * r.kos.head;
        else if (is_v) to = r.v_out + page * r.v_page + inside * r.vos.token + head * r.vos.head;
        else to = r.k_out + page * r.k_page + inside * r.kos.token + head * r.kos.head;
        u32x4 raw[2];
        h.load(from, raw);
        if (is_v) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (page >= 0 && h.there[i]) *reinterpret_cast<u32x4 *>(to + 8 * h.at[i]) = raw[i];
            continue;
        }
        float x[16];
        h.widen(raw, x);
        if (norm) {
            const float inverse = h.inverse_root(x, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] *= inverse * (is_q ? w[0][j] : w[1][j]);
        }
        h.rotate(x, 1.0f);
        if (is_q || !CACHE || page >= 0) h.store(to, x);
    }
}

// Backward.  A wave takes heads as in the forward pass, and further tokens: first all queries' heads, then all keys', so that it holds one weight and the
// gradients of one, which stay in registers and leave the block as one line of 32-bit sums.
// Bound by HBM, each of three tensors once: 8191 tokens of 2 x 16 heads of 80, 126 MB, 29.0 us, 4.3 TB/s; 12000 of 2 x 12 of 64, three axes, 111 MB, 26.5 us,
// 4.2 TB/s.  Four waves a SIMD, as many blocks as run at once; the next head's loads ahead of this one's work gained nothing.
template <class T, int G, bool NEIGHBOURS>
__global__ __launch_bounds__(256, 4) void k_rotate_back(const RotateArgs r)
{
    constexpr uint32_t PER = 64 / G;
    __shared__ float sums[4][2][16 * G];
    __shared__ __align__(16) float shared[4][2][128];
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const bool norm = r.q_weight != nullptr;
    Head<T, G, NEIGHBOURS> h(r);
    const auto pass = [&](uint32_t heads, uint32_t which, const uint16_t *x_at, const Rows &xs, const uint16_t *dy_at, const Rows &dys, uint16_t *dx_at, const Rows &dxs, const uint16_t *weight_at) {
        u32x4 weights[2];
        float dw[16] = {};
        if (norm) h.load(weight_at, weights);
        const uint32_t waves = (heads + PER - 1) / PER, shares = r.shares < waves ? r.shares : waves;
        const uint64_t step = (uint64_t)gridDim.x * 4, items = (uint64_t)r.tokens * shares;
        for (uint64_t item = (uint64_t)blockIdx.x * 4 + w; item < items; item += step) {
            const uint32_t token = (uint32_t)(item / shares), share = (uint32_t)(item % shares);
            h.angles(r, token, 0, shared[w]);
            for (uint32_t head = share * PER + lane / G; head - lane / G < heads; head += shares * PER) {
                if (head >= heads) continue;
                u32x4 raw[2], raw_d[2];
                h.load(dy_at + token * dys.token + head * dys.head, raw_d);
                if (norm) h.load(x_at + token * xs.token + head * xs.head, raw);
                asm volatile("" ::: "memory");          // the angles are read again for every head: kept, they spill other registers
                h.take(shared[w]);
                float d[16];
                h.widen(raw_d, d);
                h.rotate(d, -1.0f);
                if (norm) {
                    float x[16], weight[16];
                    h.widen(raw, x);
                    h.widen(weights, weight);
                    const float inverse = h.inverse_root(x, r);
                    float along = 0.0f;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        x[j] *= inverse;
                        dw[j] += d[j] * x[j];
                        d[j] *= weight[j];
                        along += d[j] * x[j];
                    }
                    along = h.sum(along) / (float)r.head_dim;
#pragma unroll
                    for (int j = 0; j < 16; ++j) d[j] = inverse * (d[j] - x[j] * along);
                }
                h.store(dx_at + token * dxs.token + head * dxs.head, d);
            }
        }
        if (!norm) return;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float x = dw[j];
#pragma unroll
            for (int d = G; d < 64; d <<= 1) x += __shfl_xor(x, d);
            if (lane < G) sums[w][which][16 * lane + j] = x;
        }
    };
    pass(r.heads, 0, r.q, r.qs, r.dq_out, r.dqos, r.dq, r.dqs, r.q_weight);
    pass(r.kv_heads, 1, r.k, r.ks, r.dk_out, r.dkos, r.dk, r.dks, r.k_weight);
    if (!norm) return;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 2 * 16 * G; i += 256) {
        const uint32_t n = i / (16 * G), c = i % (16 * G), chunk = c / 8 % 2, p = c / 16;
        const float x = (sums[0][n][c] + sums[1][n][c]) + (sums[2][n][c] + sums[3][n][c]);
        // lane p's chunk of the head, as Head has it
        const uint32_t chunks = r.head_dim / 8, half = NEIGHBOURS ? 0 : r.rot / 16, lanes = (chunks + 1) / 2;
        const uint32_t first = p < half ? p : half + p, at = !chunk ? first : p < half ? p + half : first + (lanes - half);
        if (p < lanes && at < chunks) r.parts[((uint64_t)blockIdx.x * 2 + n) * r.head_dim + 8 * at + c % 8] = x;
    }
}

// The weights' gradients: the blocks' lines in ascending order, 32 columns a block, 32 slices of the lines.  Up to 1024 lines: 3.9 us, a launch and two trips.
template <class T>
__global__ __launch_bounds__(1024) void k_rotate_weights(const RotateArgs r)
{
    __shared__ float slices[32][33];
    const uint32_t column = blockIdx.x * 32 + threadIdx.x % 32, slice = threadIdx.x / 32, width = 2 * r.head_dim;
    float x = 0.0f;
    if (column < width)
#pragma unroll 16
        for (uint32_t i = slice; i < r.blocks; i += 32) x += r.parts[(uint64_t)i * width + column];
    slices[slice][threadIdx.x % 32] = x;
    __syncthreads();
    if (slice || column >= width) return;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) total += slices[i][threadIdx.x];
    uint16_t *to = column < r.head_dim ? r.dq_weight + column : r.dk_weight + (column - r.head_dim);
    *reinterpret_cast<typename T::Scalar *>(to) = (typename T::Scalar)total;
}

}  // namespace mmee
