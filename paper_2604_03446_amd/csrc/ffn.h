// The gated feed-forward block and its gradient, on three kernels: products of large matrices in tiles, products of a few tokens
// with streamed weights, and sums of pieces.
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T
//   dh = dy Wd;  dg = dh u act'(g), du = dh act(g);  dx = dg Wg + du Wu;  dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//
// Products take 16-bit operands and accumulate in 32 bits.  act(g) u and the gradients through it are formed from the 32-bit
// accumulators in the product's epilogue; g and u are rounded to 16 bits only where they are kept for the backward pass, h, dg and
// du because the next product takes them as operands.
#pragma once

#include "launch.h"
#include "mfma.h"

namespace mmee {

enum { ACT_SILU = 0, ACT_GELU = 1, ACT_GELU_TANH = 2, ACT_RELU = 3, ACT_SIGMOID = 4, N_ACTS = 5 };

__device__ __forceinline__ float sigmoid_of(float x) { return 1.0f / (1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)); }

// Activation and its derivative, in 32 bits.
__device__ __forceinline__ void activate(int kind, float g, float &value, float &slope)
{
    switch (kind) {
    case ACT_SILU: {
        const float e = sigmoid_of(g);
        value = g * e;
        slope = e * (1.0f + g * (1.0f - e));
        return;
    }
    case ACT_GELU: {
        const float e = 0.5f * (1.0f + erff(0.7071067811865476f * g));
        value = g * e;
        slope = e + g * 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.7213475204444817f * g * g);
        return;
    }
    case ACT_GELU_TANH: {
        // (1 + tanh z) / 2 = sigmoid(2 z)
        const float z2 = 1.5957691216057308f * (g + 0.044715f * g * g * g), e = sigmoid_of(z2);
        value = g * e;
        slope = e + g * e * (1.0f - e) * 1.5957691216057308f * (1.0f + 0.134145f * g * g);
        return;
    }
    case ACT_RELU:
        value = __builtin_elementwise_maximum(g, 0.0f);
        slope = g > 0.0f ? 1.0f : 0.0f;
        return;
    default: {
        const float e = sigmoid_of(g);
        value = e;
        slope = e * (1.0f - e);
        return;
    }
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
};

constexpr int BK = 64;

// One thread's share of an operand's tile of ROWS x 64, by THREADS threads: registers in flight, then shared memory.
template <int ROWS, int THREADS, bool ACROSS>
struct OperandStage {
    static constexpr int CH = ACROSS ? ROWS / 8 : BK / 8, LINES = ACROSS ? BK : ROWS, LOADS = LINES * CH / THREADS, PER = THREADS / CH;
    static_assert(LOADS * THREADS == LINES * CH && PER * CH == THREADS, "a tile is dealt out evenly");
    u32x4 r[LOADS];
    uint32_t offset[LOADS];             // elements from the tile's first column (along) or line (across) on
    int chunk, line0;

    // `rows` rows from the tile's first on exist (more than none).  Rows past them repeat the last one: their results are not stored.
    // `halves`: the tile's second half begins at row `second` of the operand instead (gate and up columns of one tile).
    __device__ __forceinline__ void aim(int thread, uint32_t first, uint32_t rows, int64_t ld)
    {
        chunk = thread % CH;
        line0 = thread / CH;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t line = line0 + i * PER;
            if (ACROSS) {
                const uint32_t col = first + 8 * chunk;
                offset[i] = line * (uint32_t)ld + (col < rows ? col : rows - 8);
            } else {
                const uint32_t row = first + line;
                offset[i] = (row < rows ? line : rows - 1 - first) * (uint32_t)ld + 8 * chunk;
            }
        }
    }

    // k values k0 .. k0+63 of which `left` exist; at: the tile's first row (along) or the operand (across), at k0.
    __device__ __forceinline__ void load_one(int i, const uint16_t *at, uint32_t left)
    {
        if (left >= BK) {
            r[i] = *reinterpret_cast<const u32x4 *>(at + offset[i]);
        } else {
            const bool there = (ACROSS ? (uint32_t)(line0 + i * PER) : (uint32_t)(8 * chunk)) < left;
            r[i] = there ? *reinterpret_cast<const u32x4 *>(at + offset[i]) : u32x4{0, 0, 0, 0};
        }
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
// step's tile is stored and the one after it is on its way in registers.
template <class T, int TM, int TN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, int EPI>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_product(const ProductArgs p)
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

    auto load_a = [&](int i, uint32_t s) {
        const uint32_t seg = s >= steps1, k0 = (s - seg * steps1) * BK;
        const uint16_t *from = p.a[p.problems > 1 ? problem : seg];
        sa.load_one(i, from + (A_ACROSS ? k0 * p.lda : m0 * p.lda + k0), p.k - k0);
    };
    auto load_b = [&](int half, int i, uint32_t s) {
        const uint32_t seg = s >= steps1, k0 = (s - seg * steps1) * BK;
        const uint16_t *from = p.b[GATED ? half : p.segments > 1 ? seg : 0];
        sb[half].load_one(i, from + (B_ACROSS ? k0 * p.ldb : n0 * p.ldb + k0), p.k - k0);
    };
    constexpr int LA = decltype(sa)::LOADS, LB = OperandStage<BN, THREADS, B_ACROSS>::LOADS, HALVES = GATED ? 2 : 1, ALL = LA + HALVES * LB;
    static_assert(ALL % 4 == 0, "a quarter of the loads with each quarter of a step");
    auto load = [&](int i, uint32_t s) {
        if (i < LA) load_a(i, s);
        else load_b((i - LA) / LB, (i - LA) % LB, s);
    };
    auto store = [&](int i, u32x4 *buf) {
        if (i < LA) sa.store_one(i, buf);
        else sb[(i - LA) / LB].store_one((i - LA) % LB, buf + (TM + (i - LA) / LB * BN) * BK / 8);
    };

    f32x16 acc[MS][NS] = {};
    if (count) {
#pragma unroll
        for (int i = 0; i < ALL; ++i) load(i, step0);
#pragma unroll
        for (int i = 0; i < ALL; ++i) store(i, tiles[0]);
        if (count > 1) {
#pragma unroll
            for (int i = 0; i < ALL; ++i) load(i, step0 + 1);
        }
    }
    __syncthreads();
    for (uint32_t s = 0; s < count; ++s) {
        const u32x4 *ta = tiles[s & 1], *tb = ta + TM * BK / 8;
        u32x4 *next = tiles[(s + 1) & 1];
#pragma unroll
        for (int t = 0; t < BK / 16; ++t) {
            typename T::V8 a[MS], b[NS];
#pragma unroll
            for (int ms = 0; ms < MS; ++ms) a[ms] = operand<T, TM, A_ACROSS>(ta, (wm * MS + ms) * 32, t);
#pragma unroll
            for (int ns = 0; ns < NS; ++ns) {
                const int half = GATED ? ns / (NS / 2) : 0, block = GATED ? wn * (NS / 2) + ns % (NS / 2) : wn * NS + ns;
                b[ns] = operand<T, BN, B_ACROSS>(tb + half * BN * BK / 8, block * 32, t);
            }
            if (s + 1 < count) {
#pragma unroll
                for (int i = t * ALL / 4; i < (t + 1) * ALL / 4; ++i) store(i, next);
            }
            if (s + 2 < count) {
#pragma unroll
                for (int i = t * ALL / 4; i < (t + 1) * ALL / 4; ++i) load(i, step0 + s + 2);
            }
#pragma unroll
            for (int ms = 0; ms < MS; ++ms)
#pragma unroll
                for (int ns = 0; ns < NS; ++ns) acc[ms][ns] = T::mma(b[ns], a[ms], acc[ms][ns]);       // C^T: a lane holds one row of C
        }
        __syncthreads();
    }

#pragma unroll
    for (int ms = 0; ms < MS; ++ms) {
        const uint32_t row = m0 + (wm * MS + ms) * 32 + i32;
        if (row >= p.m) continue;
        constexpr int OUT = GATED ? NS / 2 : NS;
#pragma unroll
        for (int ns = 0; ns < OUT; ++ns)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t col = n0 + (wn * OUT + ns) * 32 + 8 * q + 4 * h;
                if (col >= p.n) continue;
                f32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = acc[ms][ns][4 * q + j];
                typedef typename T::V4 V4;
                if (EPI == EPI_STORE) {
                    if (p.splits > 1) *reinterpret_cast<f32x4 *>(p.parts + ((uint64_t)(problem * p.splits + split) * p.m + row) * p.n + col) = x;
                    else *reinterpret_cast<V4 *>(p.c[problem] + row * p.ldc + col) = __builtin_convertvector(x, V4);
                } else if (GATED) {
                    f32x4 u, y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u[j] = acc[ms][GATED ? ns + NS / 2 : ns][4 * q + j];
                        float value, slope;
                        activate(p.act, x[j], value, slope);
                        y[j] = value * u[j];
                    }
                    *reinterpret_cast<V4 *>(p.c[0] + row * p.ldc + col) = __builtin_convertvector(y, V4);
                    if (p.gate) *reinterpret_cast<V4 *>(p.gate + row * p.ld_hidden + col) = __builtin_convertvector(x, V4);
                    if (p.up) *reinterpret_cast<V4 *>(p.up + row * p.ld_hidden + col) = __builtin_convertvector(u, V4);
                } else {
                    const V4 g = *reinterpret_cast<const V4 *>(p.gate_in + row * p.ld_hidden + col), u = *reinterpret_cast<const V4 *>(p.up_in + row * p.ld_hidden + col);
                    f32x4 dg, du;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float value, slope;
                        activate(p.act, (float)g[j], value, slope);
                        dg[j] = x[j] * (float)u[j] * slope;
                        du[j] = x[j] * value;
                    }
                    *reinterpret_cast<V4 *>(p.c[0] + row * p.ldc + col) = __builtin_convertvector(dg, V4);
                    *reinterpret_cast<V4 *>(p.c[1] + row * p.ldc + col) = __builtin_convertvector(du, V4);
                }
            }
    }
}

// Sums a product's pieces in ascending order and rounds once, four values a thread.
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
    *reinterpret_cast<typename T::V4 *>(p.c[problem] + in / n4 * p.ldc + in % n4 * 4) = __builtin_convertvector(x, typename T::V4);
}

// A few tokens: C[token][n] = sum_k x[token][k] W[n][k] for up to 16 MT tokens, with the weights streamed once from memory straight
// into operands.  A block owns 16 NT rows of the weights (GATED: as many of the gate's and of the up projection's each); its eight waves
// take every eighth step of 32 along k, so that together they read 512 neighbouring bytes of a row, and are summed through
// shared memory in the order of the waves.  Nothing is shared while weights stream in and no barrier is met.
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
        typedef typename T::V4 V4;
        if (GATED) {
            const f32x4 g = y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float value, slope;
                activate(p.act, g[j], value, slope);
                y[j] = value * u[j];
            }
            if (p.gate) *reinterpret_cast<V4 *>(p.gate + token * p.ld_hidden + col) = __builtin_convertvector(g, V4);
            if (p.up) *reinterpret_cast<V4 *>(p.up + token * p.ld_hidden + col) = __builtin_convertvector(u, V4);
            *reinterpret_cast<V4 *>(p.c[0] + token * p.ldc + col) = __builtin_convertvector(y, V4);
        } else if (p.splits > 1) {
            *reinterpret_cast<f32x4 *>(p.parts + ((uint64_t)split * p.m + token) * p.n + col) = y;
        } else {
            *reinterpret_cast<V4 *>(p.c[0] + token * p.ldc + col) = __builtin_convertvector(y, V4);
        }
    }
}

}  // namespace mmee
