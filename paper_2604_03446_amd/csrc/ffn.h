// The gated feed-forward block and its gradient, on three kernels: products of large matrices in tiles, products of a few tokens
// with streamed weights, and sums of pieces.
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T
//   dh = dy Wd;  dg = dh u act'(g), du = dh act(g);  dx = dg Wg + du Wu;  dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//
// Products take 16-bit operands and accumulate in 32 bits.  act(g) u and the gradients through it are formed from the 32-bit
// accumulators in the product's epilogue; h, dg and du are rounded because the next product takes them as operands.  g and u are kept
// for the backward pass in 16 bits: dx, dWg and dWu are then 1.8 times as far from 64-bit values as one rounding of the result takes
// them (2-norm, bfloat16: 0.0031 and 0.0017).  In 32 bits it would be 1.4 times, for twice the room and 260 MB more to move at 4001 tokens of 8192.
#pragma once

#include <type_traits>

#include "launch.h"
#include "mfma.h"

namespace mmee {

enum { ACT_SILU = 0, ACT_GELU = 1, ACT_GELU_TANH = 2, ACT_RELU = 3, ACT_SIGMOID = 4, N_ACTS = 5 };

__device__ __forceinline__ float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }

// An activation and its derivative, in 32 bits.
template <int KIND>
__device__ __forceinline__ void activate(float g, float &value, float &slope)
{
    if (KIND == ACT_SILU) {
        const float e = sigmoid_of(g);
        value = g * e;
        slope = e * (1.0f + g * (1.0f - e));
    } else if (KIND == ACT_GELU) {
        // erfc(z) = t (a1 + t (a2 + ..)) exp(-z^2), t = 1 / (1 + 0.3275911 z), z >= 0, to 1.5e-7 (Abramowitz and Stegun, 7.1.26); erff
        // in its place made the epilogue of a tile of 256 x 128 results 10 us longer.
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.23164189f * __builtin_fabsf(g)), bell = __builtin_amdgcn_exp2f(-0.7213475204444817f * g * g);
        const float half = 0.5f * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f)))) * bell;
        const float e = g < 0.0f ? half : 1.0f - half;
        value = g * e;
        slope = e + g * 0.3989422804014327f * bell;
    } else if (KIND == ACT_GELU_TANH) {                 // (1 + tanh z) / 2 = sigmoid(2 z)
        const float e = sigmoid_of(1.5957691216057308f * (g + 0.044715f * g * g * g));
        const float near = __builtin_amdgcn_fmed3f(g, -16.0f, 16.0f);          // beyond it e is 0 or 1, and the square of g may be beyond 32 bits
        value = g * e;
        slope = e + near * e * (1.0f - e) * 1.5957691216057308f * (1.0f + 0.134145f * near * near);
    } else if (KIND == ACT_RELU) {
        value = __builtin_elementwise_maximum(g, 0.0f);
        slope = g > 0.0f ? 1.0f : 0.0f;
    } else {
        const float e = sigmoid_of(g);
        value = e;
        slope = e * (1.0f - e);
    }
}

// f(std::integral_constant) for the activation of a call.
template <class F>
__device__ __forceinline__ void with_activation(int kind, F f)
{
    switch (kind) {
    case ACT_SILU: f(std::integral_constant<int, ACT_SILU>()); break;
    case ACT_GELU: f(std::integral_constant<int, ACT_GELU>()); break;
    case ACT_GELU_TANH: f(std::integral_constant<int, ACT_GELU_TANH>()); break;
    case ACT_RELU: f(std::integral_constant<int, ACT_RELU>()); break;
    default: f(std::integral_constant<int, ACT_SIGMOID>()); break;
    }
}

// What a product's epilogue does with its accumulators.
enum {
    EPI_STORE = 0,      // C, or a piece's sum in 32 bits
    EPI_GATED = 1,      // gate and up columns side by side in a tile: h, and g and u where they are kept
    EPI_DGATED = 2,     // dh: dg and du from the kept g and u
};

// C[m][n] = sum_k A(m, k) B(n, k).  An operand lies along its rows, [row][k], or across, [k][row].
struct ProductArgs {
    const uint16_t *a[2], *b[2];        // segments of the sum, or problems that share the other operand
    uint16_t *c[2];
    int64_t lda, ldb, ldc;
    uint32_t m, n, k;
    uint32_t segments, problems, splits;
    uint32_t tiles_m, tiles_n;
    float *parts;                       // [problem][split][m][n]
    int act;
    const uint16_t *gate_in, *up_in;    // EPI_DGATED
    uint16_t *gate, *up;                // EPI_GATED: kept, or null
    int64_t ld_hidden;                  // of gate and up
    const float *scale;                 // float16: of dg and du, and its inverse; null: none
};

constexpr int BK = 64;

// One thread's share of an operand's tile of ROWS x 64, by THREADS threads: registers in flight, then shared memory.  What does not
// exist is asked for beyond the buffer's end and comes back as zeros, without a branch of its own.
template <int ROWS, int THREADS, bool ACROSS>
struct OperandStage {
    static constexpr int CH = ACROSS ? ROWS / 8 : BK / 8, LINES = ACROSS ? BK : ROWS, LOADS = LINES * CH / THREADS, PER = THREADS / CH;
    static_assert(LOADS * THREADS == LINES * CH && PER * CH == THREADS, "a tile is dealt out evenly");
    u32x4 r[LOADS];
    uint32_t offset[LOADS];             // bytes from the tile's first row (along) or the operand (across) on, at the step's k
    int chunk, line0;

    // `rows` rows of the operand exist, more than `first`, the tile's first.  Rows past them repeat the last one: their results are not stored.
    __device__ __forceinline__ void aim(int thread, uint32_t first, uint32_t rows, int64_t ld)
    {
        chunk = thread % CH;
        line0 = thread / CH;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t line = line0 + i * PER;
            if (ACROSS) {
                const uint32_t col = first + 8 * chunk;
                offset[i] = 2 * (line * (uint32_t)ld + (col < rows ? col : rows - 8));
            } else {
                const uint32_t row = first + line;
                offset[i] = 2 * ((row < rows ? line : rows - 1 - first) * (uint32_t)ld + 8 * chunk);
            }
        }
    }

    // k values from the step's first on, of which `left` exist; at: the tile's first row (along) or the operand (across), at that k.
    __device__ __forceinline__ void load_one(int i, __amdgpu_buffer_rsrc_t at, uint32_t left)
    {
        const bool there = (ACROSS ? (uint32_t)(line0 + i * PER) : (uint32_t)(8 * chunk)) < left;
        r[i] = __builtin_amdgcn_raw_buffer_load_b128(at, there ? offset[i] : BEYOND, 0, 0);
    }

    __device__ __forceinline__ void store_one(int i, u32x4 *tile) const { tile[chunk_at<CH>(line0 + i * PER, chunk)] = r[i]; }
};

// Operand of 32 rows `first` .. of a tile, k values 16 t ..: 8 values a lane.
template <class T, int ROWS, bool ACROSS>
__device__ __forceinline__ typename T::V8 operand(const u32x4 *tile, int first, int t)
{
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if (ACROSS) {
        constexpr int CH = ROWS / 8;
        const int i = lane & 15, g = (lane >> 4) & 1, c = first / 8 + 2 * g + ((i >> 1) & 1), line = 8 * h + (i >> 2);
        const char *base = reinterpret_cast<const char *>(tile + 16 * t * CH) + 8 * (i & 1);
        return join<T>(read_transposed(base + 16 * chunk_at<CH>(line, c)), read_transposed(base + 16 * chunk_at<CH>(line + 4, c)));
    }
    constexpr int CH = BK / 8;
    return as_operand<T>(tile[first * CH + chunk_at<CH>(lane & 31, 2 * t + h)]);
}

// A tile of TM x TN by WM x WN waves, in steps of 64 along k.  Two buffers in shared memory: while a step's products run, the next
// step's tile is stored and the one after it is on its way in registers.  A quarter of a step ahead of their use operands are
// read into registers; the step's one barrier lies ahead of its last quarter, so that the next step's first operands are there
// when it begins.  A wave of a 256 x 256 tile holds 128 x 128 results in 256 registers, for which it reads half as much from shared memory a
// product as with 64 x 64; it is then alone on its unit's quarter.
// Bound by the matrix instructions, at the clock that the card holds under them (1.8 to 2.1 GHz of 2.4).  4001 tokens, 2048 -> 8192 -> 2048, bfloat16,
// all six products: gate and up with their epilogue (h, g and u, 197 MB, leave at its end) 306 to 331 us, 0.85 PFLOP/s; y 141 to 146, 0.95; dg and du
// (g and u read, two results) 204 to 217, 0.64; dx 231 to 241 and its pieces 14, 1.1; dWg and dWu together 232 to 246, 1.1; dWd 117 to 122, 1.1.
// The instances with an epilogue (gate and up, dg and du) keep the choice of A in vector registers, so that each load of A is a loop over the
// lanes that cuts the quarter's instructions into pieces which nothing orders: with a scalar choice a training step of that size took 1138 us
// instead of 1216, the forward pass of 2048 tokens through 768 -> 3072 -> 768 52 instead of 57.
template <class T, int TM, int TN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, int EPI>
__global__ __launch_bounds__(64 * WM * WN, TM == 256 ? 1 : 2) void k_product(const ProductArgs p)
{
    constexpr int THREADS = 64 * WM * WN, MS = TM / WM / 32, NS = TN / WN / 32;        // 32 x 32 blocks of a wave
    constexpr bool GATED = EPI == EPI_GATED;
    constexpr int BN = GATED ? TN / 2 : TN;             // columns of one operand in the tile
    __shared__ u32x4 tiles[2][(TM + TN) * BK / 8];
    const int thread = threadIdx.x, wave = thread >> 6, lane = thread & 63, i32 = lane & 31, h = lane >> 5;
    const int wm = wave % WM, wn = wave / WM;

    // Neighbouring blocks of a die take 8 rows of tiles at a time: its L2 serves their common operands.
    uint32_t at = by_die(blockIdx.x, gridDim.x);
    const uint32_t per = p.tiles_m * p.tiles_n;
    const uint32_t problem = at / (per * p.splits);
    at -= problem * per * p.splits;
    const uint32_t split = at / per;
    at -= split * per;
    const uint32_t band = at / (8 * p.tiles_n), tall = p.tiles_m - 8 * band < 8 ? p.tiles_m - 8 * band : 8;
    at -= band * 8 * p.tiles_n;
    const uint32_t m0 = (8 * band + at % tall) * TM, n0 = at / tall * BN;

    OperandStage<TM, THREADS, A_ACROSS> sa;
    OperandStage<BN, THREADS, B_ACROSS> sb[GATED ? 2 : 1];
    sa.aim(thread, m0, p.m, p.lda);
    sb[0].aim(thread, n0, p.n, p.ldb);
    if (GATED) sb[GATED].aim(thread, n0, p.n, p.ldb);

    const uint32_t steps1 = (p.k + BK - 1) / BK, steps = steps1 * p.segments, each = (steps + p.splits - 1) / p.splits;
    const uint32_t step0 = split * each < steps ? split * each : steps, count = step0 + each < steps ? each : steps - step0;

    constexpr int LA = decltype(sa)::LOADS, LB = OperandStage<BN, THREADS, B_ACROSS>::LOADS, HALVES = GATED ? 2 : 1, ALL = LA + HALVES * LB;
    // Loads first .. last-1 of a step; steps past the piece's last load nothing.
    auto load = [&](int first, int last, uint32_t s) {
        const uint32_t step = step0 + s, seg = step >= steps1, k0 = (step - seg * steps1) * BK, left = s < count ? p.k - k0 : 0;
        const auto at_a = buffer_at((p.problems > 1 ? problem : seg) ? p.a[1] + (A_ACROSS ? k0 * p.lda : m0 * p.lda + k0) : p.a[0] + (A_ACROSS ? k0 * p.lda : m0 * p.lda + k0));
        const int64_t b_at = B_ACROSS ? k0 * p.ldb : n0 * p.ldb + k0;
        const auto at_b = buffer_at((!GATED && p.segments > 1 && seg ? p.b[1] : p.b[0]) + b_at), at_b2 = buffer_at(p.b[1] + b_at);
#pragma unroll
        for (int i = first; i < last; ++i) {
            if (i < LA) sa.load_one(i, at_a, left);
            else if (i < LA + LB) sb[0].load_one(i - LA, at_b, left);
            else sb[HALVES - 1].load_one(i - LA - LB, at_b2, left);
        }
    };
    auto store = [&](int first, int last, u32x4 *buf) {
#pragma unroll
        for (int i = first; i < last; ++i) {
            if (i < LA) sa.store_one(i, buf);
            else sb[(i - LA) / LB].store_one((i - LA) % LB, buf + (TM + (i - LA) / LB * BN) * BK / 8);
        }
    };
    typename T::V8 a[2][MS], b[2][NS];
    auto read = [&](int to, const u32x4 *tile, int t) {
#pragma unroll
        for (int ms = 0; ms < MS; ++ms) a[to][ms] = operand<T, TM, A_ACROSS>(tile, (wm * MS + ms) * 32, t);
#pragma unroll
        for (int ns = 0; ns < NS; ++ns) {
            const int half = GATED ? ns / (NS / 2) : 0, block = GATED ? wn * (NS / 2) + ns % (NS / 2) : wn * NS + ns;
            b[to][ns] = operand<T, BN, B_ACROSS>(tile + (TM + half * BN) * BK / 8, block * 32, t);
        }
    };

    f32x16 acc[MS][NS] = {};
    load(0, ALL, 0);
    store(0, ALL, tiles[0]);
    load(0, ALL, 1);
    __syncthreads();
    read(0, tiles[0], 0);
    for (uint32_t s = 0; s < count; ++s) {
        const u32x4 *now = tiles[s & 1];
        u32x4 *next = tiles[(s + 1) & 1];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t == 3) __syncthreads();                // the next tile is complete, and this one's operands are all in registers
            read((t + 1) & 1, t < 3 ? now : next, (t + 1) & 3);
            if (t < 3) {
                store(t * ALL / 3, (t + 1) * ALL / 3, next);
                load(t * ALL / 3, (t + 1) * ALL / 3, s + 2);
            }
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int ns = 0; ns < NS; ++ns) acc[ms][ns] = T::mma(b[t & 1][ns], a[t & 1][ms], acc[ms][ns]);       // C^T: a lane holds one row of C
            // The order of a quarter: a product after every operand read, then after every store and load.  (Reads spread over the whole
            // quarter, or stores between them: 2 to 13 % slower.  Tiles straight to shared memory, which leaves loads one step instead of two to
            // arrive: h of a prompt 7 to 13 % faster, y, dx and the weights' gradients 9 to 30 % slower.)
            constexpr int READS = MS * (A_ACROSS ? 2 : 1) + NS * (B_ACROSS ? 2 : 1), PRODUCTS = MS * NS;
#pragma unroll
            for (int i = 0; i < PRODUCTS / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, (READS + PRODUCTS / 2 - 1) / (PRODUCTS / 2), 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
#pragma unroll
            for (int i = 0; i < PRODUCTS / 2; ++i) {
                if (t < 3) {
                    __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();

    // Results go through the wave's share of the tiles' memory, 32 rows at a time, so that lanes next to each other hold eight
    // columns each of one row: whole lines are read and written.  What the epilogue reads is asked for 32 rows ahead.
    constexpr int COLS = 32 * NS, C4 = COLS / 4, OUT = GATED ? COLS / 2 : COLS, PER_ROW = OUT / 8, ROWS = 64 / PER_ROW, PASSES = 32 / ROWS;
    constexpr bool DGATED = EPI == EPI_DGATED;
    static_assert(sizeof(tiles) >= sizeof(float) * WM * WN * 32 * COLS, "32 rows of every wave fit");
    typedef typename T::V8 V8;
    f32x4 *mine = reinterpret_cast<f32x4 *>(&tiles[0][0]) + wave * 32 * C4;
    const int c8 = lane % PER_ROW, r0 = lane / PER_ROW;
    const uint32_t col = n0 + wn * OUT + 8 * c8, rows0 = m0 + wm * MS * 32 + r0;
    const float times = NARROW<T> && !GATED && p.scale ? p.scale[DGATED ? 0 : 1] : 1.0f;
    const bool column = col < p.n;
    V8 kept[2][DGATED ? PASSES : 1];                    // g and u
    auto ask = [&](int ms) {
        if (!DGATED) return;
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            const uint32_t row = rows0 + ms * 32 + pass * ROWS;
            const uint64_t at = (uint64_t)(row < p.m ? row : p.m - 1) * p.ld_hidden + (column ? col : 0);
            kept[0][DGATED ? pass : 0] = *reinterpret_cast<const V8 *>(p.gate_in + at);
            kept[1][DGATED ? pass : 0] = *reinterpret_cast<const V8 *>(p.up_in + at);
        }
    };
    auto take = [&](int in, int c) {
        const f32x4 lo = mine[in * C4 + (c ^ (in & (C4 - 1)))], hi = mine[in * C4 + ((c + 1) ^ (in & (C4 - 1)))];
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    ask(0);
#pragma unroll 1
    for (int ms = 0; ms < MS; ++ms) {
        wave_sync();
#pragma unroll
        for (int which = 0; which < MS; ++which)
            if (which == ms) {
#pragma unroll
                for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16 &from = acc[which][ns];
                        mine[i32 * C4 + ((8 * ns + 2 * q + h) ^ (i32 & (C4 - 1)))] = f32x4{from[4 * q], from[4 * q + 1], from[4 * q + 2], from[4 * q + 3]};
                    }
            }
        wave_sync();
        V8 g[DGATED ? PASSES : 1], u[DGATED ? PASSES : 1];
        if (DGATED) {
#pragma unroll
            for (int pass = 0; pass < PASSES; ++pass) {
                g[DGATED ? pass : 0] = kept[0][DGATED ? pass : 0];
                u[DGATED ? pass : 0] = kept[1][DGATED ? pass : 0];
            }
            ask(ms + 1 < MS ? ms + 1 : ms);
        }
        const uint32_t row0 = rows0 + ms * 32;
        if (EPI == EPI_STORE) {
#pragma unroll
            for (int pass = 0; pass < PASSES; ++pass) {
                const uint32_t row = row0 + pass * ROWS;
                const f32x8 x = take(pass * ROWS + r0, 2 * c8);
                if (row >= p.m || !column) continue;
                if (p.splits > 1) *reinterpret_cast<f32x8 *>(p.parts + ((uint64_t)(problem * p.splits + split) * p.m + row) * p.n + col) = x;
                else *reinterpret_cast<V8 *>(p.c[problem] + row * p.ldc + col) = __builtin_convertvector(NARROW<T> ? x * times : x, V8);
            }
        } else {
            with_activation(p.act, [&](auto kind) {
#pragma unroll
                for (int pass = 0; pass < PASSES; ++pass) {
                    const uint32_t row = row0 + pass * ROWS;
                    f32x8 x = take(pass * ROWS + r0, 2 * c8);
                    if (NARROW<T> && DGATED) x *= times;
                    f32x8 value, slope;
                    if (GATED) {
                        const f32x8 up = take(pass * ROWS + r0, 2 * c8 + C4 / 2);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float y, unused;
                            activate<kind.value>(x[j], y, unused);
                            value[j] = y * up[j];
                        }
                        if (row >= p.m || !column) continue;
                        *reinterpret_cast<V8 *>(p.c[0] + row * p.ldc + col) = __builtin_convertvector(value, V8);
                        if (p.gate) *reinterpret_cast<V8 *>(p.gate + row * p.ld_hidden + col) = __builtin_convertvector(x, V8);
                        if (p.up) *reinterpret_cast<V8 *>(p.up + row * p.ld_hidden + col) = __builtin_convertvector(up, V8);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float y, dy;
                            activate<kind.value>((float)g[DGATED ? pass : 0][j], y, dy);
                            value[j] = x[j] * y;
                            slope[j] = x[j] * (float)u[DGATED ? pass : 0][j] * dy;
                        }
                        if (row >= p.m || !column) continue;
                        *reinterpret_cast<V8 *>(p.c[0] + row * p.ldc + col) = __builtin_convertvector(slope, V8);
                        *reinterpret_cast<V8 *>(p.c[1] + row * p.ldc + col) = __builtin_convertvector(value, V8);
                    }
                }
            });
        }
    }
}

// Sums a product's pieces in ascending order and rounds once, four values a thread.  Bound by memory: two pieces of 4001 x 2048, 82 MB
// with the result: 14 us, 5.8 TB/s (some of it from the last level of cache); in small calls a launch, 2 us.
template <class T>
__global__ __launch_bounds__(256) void k_sum_parts(const ProductArgs p)
{
    const uint64_t n4 = p.n / 4, per = n4 * p.m, at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= per * p.problems) return;
    const uint32_t problem = (uint32_t)(at / per);
    const uint64_t in = at - problem * per;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t s = 0; s < p.splits; ++s) x += *reinterpret_cast<const f32x4 *>(p.parts + ((problem * p.splits + s) * per + in) * 4);
    if (NARROW<T> && p.scale) x *= p.scale[1];
    *reinterpret_cast<typename T::V4 *>(p.c[problem] + in / n4 * p.ldc + in % n4 * 4) = __builtin_convertvector(x, typename T::V4);
}

// Float16's dg and du.  They are the next products' operands, and with the gradients of a long mean they lie below the type's normal numbers
// (6e-5), where rounding is no longer relative, while the weights' gradients, sums over the tokens, lie well above.  So both are multiplied by a power of two of the call's
// own, which is divided out of the 32-bit sums.  |dg| and |du| are at most max_t |dy_t| max_f |wd_f| max(1.13 |u|, |act(g)|) (2-norms of dy's
// rows and of Wd's columns, as dh is their product; act' is at most 1.13, |act(g)| at most |g|, or 1): the power takes this bound to 2^14 .. 2^15, so that nothing
// overflows.  The typical value lies about sqrt(out_dim) and the outliers' ratios below it: of 2^29 between the bound and the last normal number
// most is left.  A token whose gradient is far below the largest one's (2^-15 and less) gets a dx of fewer bits.
struct BoundArgs {
    const uint16_t *dy, *w_down, *gate, *up;
    int64_t ld_dy, ld_down;
    uint32_t rows, hidden, out;
    uint32_t row_blocks, kept_blocks, strips, chunks;   // blocks for dy's rows, for g and u, for 64 rows of 512 of Wd's columns each
    int act;
    float *parts;                       // what they found: [row_blocks], [kept_blocks][2], [chunks][strips]
    float *scale;
};

__device__ __forceinline__ float finite_or_zero(float x) { return x < INFINITY ? x : 0.0f; }      // (NaN neither)

template <class T>
__device__ __forceinline__ f32x8 eight(const uint16_t *p) { return __builtin_convertvector(*reinterpret_cast<const typename T::V8 *>(p), f32x8); }

// Bound by memory: 4001 tokens, 2048 -> 8192 -> 2048: 34 us for 181 MB, 5.3 TB/s.  With k_grad_scale's 4 us, the latency of its loads, 3 % of that
// training step; 64 tokens through 4096 -> 12288 -> 4096, most of it Wd's, or 300 through 768 -> 3072 -> 768: 10 %.
template <class T>
__global__ __launch_bounds__(256) void k_grad_bounds(const BoundArgs p)
{
    __shared__ float found[2][4];
    __shared__ float squares[4][512];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t at = blockIdx.x;
    float *out = p.parts;
    float most = 0.0f, second = 0.0f;
    uint32_t kinds = 1;
    if (at < p.row_blocks) {                            // squares of dy's rows, a wave each
        out += at;
        for (uint64_t row = 4ull * at + wave; row < p.rows; row += 4ull * p.row_blocks) {
            float sum = 0.0f;
            for (uint32_t c = 8 * lane; c < p.out; c += 512) {
                const f32x8 x = eight<T>(p.dy + row * p.ld_dy + c);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
            most = __builtin_fmaxf(most, finite_or_zero(sum));
        }
    } else if ((at -= p.row_blocks) < p.kept_blocks) {  // |g| and |u|
        out += p.row_blocks + 2 * at;
        kinds = 2;
        const uint64_t all = (uint64_t)p.rows * p.hidden, stride = 2048ull * p.kept_blocks;
        for (uint64_t i = 2048ull * at + 8 * threadIdx.x; i < all; i += stride) {
            const f32x8 g = eight<T>(p.gate + i), u = eight<T>(p.up + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                most = __builtin_fmaxf(most, finite_or_zero(__builtin_fabsf(g[j])));
                second = __builtin_fmaxf(second, finite_or_zero(__builtin_fabsf(u[j])));
            }
        }
    } else {                                            // squares of 64 rows of Wd's columns, 512 of them
        at -= p.kept_blocks;
        out += p.row_blocks + 2 * p.kept_blocks + at;
        const uint32_t col = at % p.strips * 512 + 8 * lane, row0 = at / p.strips * 64;
        f32x8 sum = {};
        if (col < p.hidden) {
#pragma unroll 4
            for (uint32_t row = row0 + wave; row < row0 + 64 && row < p.out; row += 4) {
                const f32x8 x = eight<T>(p.w_down + row * p.ld_down + col);
                sum += x * x;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) squares[wave][8 * lane + j] = sum[j];
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < 512; c += 256)
            most = __builtin_fmaxf(most, finite_or_zero(squares[0][c] + squares[1][c] + squares[2][c] + squares[3][c]));
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        most = __builtin_fmaxf(most, __shfl_xor(most, d));
        second = __builtin_fmaxf(second, __shfl_xor(second, d));
    }
    if (lane == 0) {
        found[0][wave] = most;
        found[1][wave] = second;
    }
    __syncthreads();
    if (threadIdx.x < kinds) {
        const float *f = found[threadIdx.x];
        out[threadIdx.x] = __builtin_fmaxf(__builtin_fmaxf(f[0], f[1]), __builtin_fmaxf(f[2], f[3]));
    }
}

// The power of two from what the blocks found, by one block.  The largest column of Wd is at most the sum of the chunks' largest.
__global__ __launch_bounds__(1024) void k_grad_scale(const BoundArgs p)
{
    __shared__ float found[4][16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float *kept = p.parts + p.row_blocks, *w = kept + 2 * p.kept_blocks;
    float most[4] = {};                                 // dy's rows, g, u; Wd: a sum
    for (uint32_t i = threadIdx.x; i < p.row_blocks; i += 1024) most[0] = __builtin_fmaxf(most[0], p.parts[i]);
    for (uint32_t i = threadIdx.x; i < p.kept_blocks; i += 1024) {
        most[1] = __builtin_fmaxf(most[1], kept[2 * i]);
        most[2] = __builtin_fmaxf(most[2], kept[2 * i + 1]);
    }
    for (uint32_t c = threadIdx.x; c < p.chunks; c += 1024) {
        float strip = 0.0f;
#pragma unroll 4
        for (uint32_t s = 0; s < p.strips; ++s) strip = __builtin_fmaxf(strip, w[(uint64_t)c * p.strips + s]);
        most[3] += strip;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
#pragma unroll
        for (int k = 0; k < 3; ++k) most[k] = __builtin_fmaxf(most[k], __shfl_xor(most[k], d));
        most[3] += __shfl_xor(most[3], d);
    }
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) found[k][wave] = most[k];
    }
    __syncthreads();
    if (threadIdx.x) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int k = 0; k < 3; ++k) most[k] = __builtin_fmaxf(i ? most[k] : 0.0f, found[k][i]);
        most[3] = (i ? most[3] : 0.0f) + found[3][i];
    }
    const float bound = __builtin_sqrtf(most[0]) * __builtin_sqrtf(most[3]) * __builtin_fmaxf(1.13f * most[2], p.act == ACT_SIGMOID ? 1.0f : most[1]);
    const int power = bound > 0.0f ? 15 - __builtin_amdgcn_frexp_expf(bound) : 0;        // (the bound lies between 2^-72 and 2^72)
    p.scale[0] = __builtin_ldexpf(1.0f, power);
    p.scale[1] = __builtin_ldexpf(1.0f, -power);
}

// Four columns of a token's results; of a gated product from g and u.
template <class T, bool GATED>
__device__ __forceinline__ void store_tokens(const ProductArgs &p, uint32_t token, uint32_t col, uint32_t split, f32x4 y, f32x4 u)
{
    typedef typename T::V4 V4;
    if (GATED) {
        const f32x4 g = y;
        with_activation(p.act, [&](auto kind) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float value, unused;
                activate<kind.value>(g[j], value, unused);
                y[j] = value * u[j];
            }
        });
        if (p.gate) *reinterpret_cast<V4 *>(p.gate + token * p.ld_hidden + col) = __builtin_convertvector(g, V4);
        if (p.up) *reinterpret_cast<V4 *>(p.up + token * p.ld_hidden + col) = __builtin_convertvector(u, V4);
        *reinterpret_cast<V4 *>(p.c[0] + token * p.ldc + col) = __builtin_convertvector(y, V4);
    } else if (p.splits > 1) {
        *reinterpret_cast<f32x4 *>(p.parts + ((uint64_t)split * p.m + token) * p.n + col) = y;
    } else {
        *reinterpret_cast<V4 *>(p.c[0] + token * p.ldc + col) = __builtin_convertvector(y, V4);
    }
}

// A few tokens: C[token][n] = sum_k x[token][k] W[n][k] for up to 16 MT tokens, with the weights streamed once from memory straight
// into operands.  A block owns 16 NT rows of the weights (GATED: as many of the gate's and of the up projection's each); its eight waves
// take every eighth step of 32 along k, so that together they read 512 neighbouring bytes of a row, and are summed through
// shared memory in the order of the waves.  Nothing is shared while weights stream in and no barrier is met.
// Bound by HBM, and for small weights by latency: one token, 768 -> 3072 -> 768: 4.8 us for 9.4 MB and 4.0 for 4.7, about a launch and one
// trip to memory each.
template <class T, int MT, int NT, bool GATED>
__global__ __launch_bounds__(512, 2) void k_tokens(const ProductArgs p)
{
    constexpr int WAVES = 8, R = GATED ? 2 * NT : NT, UNROLL = 4;
    __shared__ f32x4 sums[WAVES][R * MT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane & 15, kg = lane >> 4;
    uint32_t at = by_die(blockIdx.x, gridDim.x);
    const uint32_t split = at % p.splits, n0 = at / p.splits * 16 * NT;
    const uint32_t steps = (p.k + 31) / 32, each = (steps + p.splits - 1) / p.splits;
    const uint32_t step0 = split * each < steps ? split * each : steps, count = step0 + each < steps ? each : steps - step0;

    const uint16_t *w[R], *x[MT];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = n0 + 16 * (r % NT) + i;
        w[r] = p.b[r / NT] + (int64_t)(row < p.n ? row : p.n - 1) * p.ldb + 8 * kg;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = p.a[0] + (int64_t)(16 * m + i < p.m ? 16 * m + i : p.m - 1) * p.lda + 8 * kg;

    f32x4 acc[R][MT] = {};
    auto run = [&](uint32_t s, bool edge) {             // one step: 32 values of k
        const uint32_t k0 = (step0 + s) * 32;
        const bool there = !edge || k0 + 8 * kg < p.k;
        u32x4 a[MT], b[R];
#pragma unroll
        for (int r = 0; r < R; ++r) b[r] = there ? *reinterpret_cast<const u32x4 *>(w[r] + k0) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < MT; ++m) a[m] = there ? *reinterpret_cast<const u32x4 *>(x[m] + k0) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[r][m] = T::mma(as_operand<T>(b[r]), as_operand<T>(a[m]), acc[r][m]);
    };
    const uint32_t inner = (step0 + count) * 32 <= p.k ? count : count - 1;             // steps that lie inside k as a whole
    uint32_t s = wave;
    for (; s + (UNROLL - 1) * WAVES < inner; s += UNROLL * WAVES) {
        u32x4 a[UNROLL][MT], b[UNROLL][R];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint32_t k0 = (step0 + s + u * WAVES) * 32;
#pragma unroll
            for (int r = 0; r < R; ++r) b[u][r] = *reinterpret_cast<const u32x4 *>(w[r] + k0);
#pragma unroll
            for (int m = 0; m < MT; ++m) a[u][m] = *reinterpret_cast<const u32x4 *>(x[m] + k0);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[r][m] = T::mma(as_operand<T>(b[u][r]), as_operand<T>(a[u][m]), acc[r][m]);
    }
    for (; s < count; s += WAVES) run(s, s >= inner);

#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) sums[wave][r * MT + m][lane] = acc[r][m];
    __syncthreads();
    // block (r, m) of 16 x 16 results: lane holds token 16 m + i, columns 16 r + 4 kg + {0..3}
    for (int job = wave; job < NT * MT; job += WAVES) {
        const int r = job / MT, m = job % MT;
        f32x4 y = {0, 0, 0, 0}, u = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            y += sums[v][r * MT + m][lane];
            if (GATED) u += sums[v][((GATED ? NT : 0) + r) * MT + m][lane];
        }
        const uint32_t token = 16 * m + i, col = n0 + 16 * r + 4 * kg;
        if (token >= p.m || col >= p.n) continue;
        store_tokens<T, GATED>(p, token, col, split, y, u);
    }
}

// As k_tokens, for more than 8 tokens, whose operands would be read as often as the weights': WR waves with 16 NT rows each share a
// chunk of 64 values of k of all tokens in shared memory, 8 / WR such groups take every (8 / WR)-th chunk.  Weights are asked for two chunks ahead,
// straight into operands; the tokens' next chunk is on its way meanwhile.  Bound by HBM: 37 tokens, 4096 -> 12288 -> 4096: 45 us for 201 MB, 4.5 TB/s
// (a copy reaches 4.7), and 25 for 101 MB with its pieces, 4.0.  The wave's number is in vector registers here, and with it the buffers that loads
// name: each load is a loop over the lanes (both products took 71 us with it in a scalar one, 75 as it is).
template <class T, int MT, int NT, int WR, bool GATED>
__global__ __launch_bounds__(512, 2) void k_tokens_shared(const ProductArgs p)
{
    constexpr int WAVES = 8, WK = WAVES / WR, R = GATED ? 2 * NT : NT, CH = BK / 8, TOKENS = 16 * MT, GT = 64 * WR;
    constexpr int LOADS = (TOKENS * CH + GT - 1) / GT, CHUNKS = WK * 2 * TOKENS * CH, SUMS = WK > 1 ? WAVES * R * MT * 64 : 0;
    __shared__ u32x4 memory[CHUNKS > SUMS ? CHUNKS : SUMS];
    const int wave = threadIdx.x >> 6, wr = wave % WR, wk = wave / WR, lane = threadIdx.x & 63, i = lane & 15, kg = lane >> 4, thread = threadIdx.x % GT;
    uint32_t at = by_die(blockIdx.x, gridDim.x);
    const uint32_t split = at % p.splits, n0 = at / p.splits * 16 * NT * WR + wr * 16 * NT;
    const uint32_t chunks = (p.k + BK - 1) / BK, each = (chunks + p.splits - 1) / p.splits;
    const uint32_t chunk0 = split * each < chunks ? split * each : chunks, mine = chunk0 + each < chunks ? each : chunks - chunk0, count = (mine + WK - 1) / WK;

    // what does not exist is asked for beyond the buffer's end
    uint32_t w[R], x[LOADS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = 16 * (r % NT) + i;
        w[r] = 2 * ((n0 + row < p.n ? row : 0) * (uint32_t)p.ldb + 8 * kg);
    }
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
        const uint32_t token = (thread + l * GT) / CH;
        x[l] = token < p.m ? 2 * (token * (uint32_t)p.lda + 8 * (thread % CH)) : BEYOND;
    }
    u32x4 wait[2][R][2], next[LOADS];
    auto ask_weights = [&](u32x4 (&to)[R][2], uint32_t s) {
        const uint32_t k0 = s < count && wk + s * WK < mine ? (chunk0 + wk + s * WK) * BK : p.k, left = p.k - k0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const auto from = buffer_at(p.b[r / NT] + (int64_t)(n0 < p.n ? n0 : 0) * p.ldb + k0);
#pragma unroll
            for (int t = 0; t < 2; ++t) to[r][t] = __builtin_amdgcn_raw_buffer_load_b128(from, (uint32_t)(32 * t + 8 * kg) < left ? w[r] + 64 * t : BEYOND, 0, 0);
        }
    };
    auto ask_tokens = [&](uint32_t s) {
        const uint32_t k0 = s < count && wk + s * WK < mine ? (chunk0 + wk + s * WK) * BK : p.k, left = p.k - k0;
        const auto from = buffer_at(p.a[0] + k0);
#pragma unroll
        for (int l = 0; l < LOADS; ++l) next[l] = __builtin_amdgcn_raw_buffer_load_b128(from, (uint32_t)(8 * (thread % CH)) < left ? x[l] : BEYOND, 0, 0);
    };
    auto put_tokens = [&](uint32_t s) {
        u32x4 *tile = memory + (wk * 2 + (s & 1)) * TOKENS * CH;
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
            const int token = (thread + l * GT) / CH;
            if (TOKENS * CH % GT == 0 || token < TOKENS) tile[chunk_at<CH>(token, thread % CH)] = next[l];
        }
    };
    f32x4 acc[R][MT] = {};
    auto step = [&](uint32_t s, u32x4 (&now)[R][2]) {
        const u32x4 *tile = memory + (wk * 2 + (s & 1)) * TOKENS * CH;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const auto tokens = as_operand<T>(tile[chunk_at<CH>(16 * m + i, 4 * t + kg)]);
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r][m] = T::mma(as_operand<T>(now[r][t]), tokens, acc[r][m]);
            }
        put_tokens(s + 1);
        ask_weights(now, s + 2);
        ask_tokens(s + 2);
        __syncthreads();
    };
    ask_tokens(0);
    ask_weights(wait[0], 0);
    ask_weights(wait[1], 1);
    put_tokens(0);
    ask_tokens(1);
    __syncthreads();
    for (uint32_t s = 0; s < count; s += 2) {           // (one step past an odd count works on zeros)
        step(s, wait[0]);
        step(s + 1, wait[1]);
    }

    f32x4 *sums = reinterpret_cast<f32x4 *>(memory);
    if (WK > 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < MT; ++m) sums[(wave * R * MT + r * MT + m) * 64 + lane] = acc[r][m];
        __syncthreads();
    }
    // block (r, m) of 16 x 16 results of row group wr: lane holds token 16 m + i, columns 16 r + 4 kg + {0..3}; the groups' waves share them
#pragma unroll
    for (int job = 0; job < NT * MT; ++job) {
        if (job % WK != wk) continue;
        const int r = job / MT, m = job % MT;
        f32x4 y = acc[r][m], u = acc[GATED ? NT + r : r][m];
        if (WK > 1) {
            y = u = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int v = 0; v < WK; ++v) {
                y += sums[((v * WR + wr) * R * MT + r * MT + m) * 64 + lane];
                if (GATED) u += sums[((v * WR + wr) * R * MT + ((GATED ? NT : 0) + r) * MT + m) * 64 + lane];
            }
        }
        const uint32_t token = 16 * m + i, col = n0 + 16 * r + 4 * kg;
        if (token >= p.m || col >= p.n) continue;
        store_tokens<T, GATED>(p, token, col, split, y, u);
    }
}

}  // namespace mmee
