// Attention of packed prompts: sequences of different lengths one behind the other, each row over its own sequence's keys, all of them or those
// up to its own.  Formulas, the folding of query heads into rows, the transposed scores and what is rounded are those of attention.h.
//
// A sequence's rows (for dK and dV its keys) are cut into tiles of a block each.  The host does not know the lengths: it launches as many blocks as any
// lengths can need, and those without a tile end at once.  Which tile a block has comes from the starts alone,
//   by slots: tile t of sequence b has slot (first row of b) / TILE + b + t, which differ whatever the lengths; or
//   by a plan that k_prompt_plan makes of the starts: the longest tiles first, whatever sequence they are of, so that the short ones fill up the end, and
//   from tiles that are longer than a unit's share pieces of that length cut off, which are joined afterwards.  It costs a launch, 5 to 8 us.  (Planned by
//   every block for itself it cost each 1 to 2 us, and blocks without a tile between those with one left some shader engines idle.)
//
// Times are of one MI355X, the least of 20 passes; matrix products hold its clock at 1.85 to 2.05 GHz.  `busy` is the share of a unit's busy cycles in which
// its matrix instructions run.  Registers that are spilled: k_prompt_forward with 64 values a head 2 (four blocks a unit); k_prompt_dq with four
// waves 4 (float16, 128 a head), 1 (float16, 64) and 8 (bfloat16, 128); k_prompt_dkv with 128 a head and four waves 4 (float16) and 2 (bfloat16), with
// eight 8 (float16); k_prompt_dkv_wide 16, outside its loop.
#pragma once

#include "attention.h"
#include "sequences.h"

namespace mmee {

struct PromptArgs {
    AttnArgs a;                 // batch 1, q_len: all tokens, rows: of all tokens, kv_len: all keys
    const int32_t *q_starts, *kv_starts;
    uint32_t seqs, slots;       // slots: of tiles, or of a plan's entries, of every head
    uint32_t parts;             // pieces of cut tiles, at most, of every head
    float *lse2;                // backward, bfloat16: [kv_head][row], in powers of two, infinite where a row sees nothing
    const uint32_t *plan;       // or null
    bool causal;
    bool dies;                  // heads are dealt out to the dies, whose L2 then holds their keys
};

// A plan: words 0 and 1 the numbers of entries and of tiles that were cut, the entries, the numbers of the cut tiles' first entries (parts / 2 at most).  An
// entry:
constexpr uint32_t ENTRIES = 8, ENTRY = 12;             // words: q0, m, k0, n, index, step0, count, piece, pieces, number of the tile's first piece, two unused

// Keys 0 .. of its sequence that a token sees.
__device__ __forceinline__ uint32_t limit_of(const PromptArgs &p, uint32_t m, uint32_t n, uint32_t token)
{
    return p.causal ? (uint32_t)within((int64_t)token + 1 + n - m, 0, n) : n;
}

// The first row that sees a key, which may lie before the sequence's first or behind its last one.
__device__ __forceinline__ int first_row(const PromptArgs &p, uint32_t m, uint32_t n, uint32_t key)
{
    return p.causal ? (int)within(((int64_t)key + m - n) * p.a.group, -(1 << 29), (int64_t)m * p.a.group) : 0;
}

// Sequence `seq`: m tokens from q0 on over n keys from k0 on.
struct Sequence {
    uint32_t q0, m, k0, n;
    __device__ __forceinline__ Sequence(const PromptArgs &p, uint32_t seq)
    {
        q0 = (uint32_t)within(p.q_starts[seq], 0, p.a.q_len);
        m = (uint32_t)within(p.q_starts[seq + 1], q0, p.a.q_len) - q0;
        k0 = (uint32_t)within(p.kv_starts[seq], 0, p.a.kv_len);
        n = (uint32_t)within(p.kv_starts[seq + 1], k0, p.a.kv_len) - k0;
    }
    // Rows, or keys, that are cut into tiles; steps of a tile of them: of `step` keys, or rows.
    __device__ __forceinline__ uint32_t lines(const PromptArgs &p, bool keys) const { return keys ? n : m * p.a.group; }
    __device__ __forceinline__ uint32_t steps(const PromptArgs &p, bool keys, uint32_t tile, uint32_t step, uint32_t index) const
    {
        const uint32_t rows = m * p.a.group;
        if (keys) {
            const int begin = first_row(p, m, n, index * tile);
            return (rows - (begin < 0 ? 0 : begin) + step - 1) / step;
        }
        const uint32_t behind = (index + 1) * tile < rows ? (index + 1) * tile : rows;
        return (limit_of(p, m, n, token_of(p.a, behind - 1)) + step - 1) / step;
    }
};

// A block's tile: rows (or, with KEYS, keys) index * TILE .. of a sequence, and the steps step0 .. of STEP keys (or rows) that are the block's piece of it.
template <uint32_t TILE, uint32_t STEP, bool KEYS>
struct Tile {
    uint32_t index, q0, m, k0, n, kvh, piece = 0, pieces = 1, first_part = 0, step0 = 0, count = 0;
    bool there;

    // at: place among heads and slots; with CUT: among heads and the tiles that were cut.
    template <bool CUT = false>
    __device__ __forceinline__ Tile(const PromptArgs &p, uint32_t at, std::integral_constant<bool, CUT> = {})
    {
        if (CUT) {
            const uint32_t most = p.parts / 2;
            kvh = at / most;
            there = at % most < p.plan[1];
            if (there) take(p.plan + ENTRIES + ENTRY * p.plan[ENTRIES + ENTRY * p.slots + at % most]);
            return;
        }
        kvh = p.dies ? at / p.slots : at % p.a.kv_heads;
        const uint32_t slot = p.dies ? at % p.slots : at / p.a.kv_heads;
        if (p.plan) {
            const uint32_t entries = p.plan[0];
            take(p.plan + ENTRIES + ENTRY * slot);      // (whatever it holds: one trip to memory for both)
            there = slot < entries;
            return;
        }
        const int32_t *starts = KEYS ? p.kv_starts : p.q_starts;
        const uint32_t tokens = KEYS ? p.a.kv_len : p.a.q_len, each = KEYS ? 1 : p.a.group;
        const auto slot_of = [&](uint32_t i) { return (int64_t)((uint32_t)within(starts[i], 0, tokens) * each / TILE + i); };
        const int seq = __builtin_amdgcn_readfirstlane(last_at_most(p.seqs, slot, slot_of));
        there = false;
        if (seq < 0) return;
        const Sequence s(p, seq);
        q0 = s.q0;
        m = s.m;
        k0 = s.k0;
        n = s.n;
        index = slot - (uint32_t)slot_of(seq);
        there = index < (s.lines(p, KEYS) + TILE - 1) / TILE;
        if (there) count = s.steps(p, KEYS, TILE, STEP, index);
    }

    __device__ __forceinline__ void take(const uint32_t *entry)
    {
        q0 = entry[0];
        m = entry[1];
        k0 = entry[2];
        n = entry[3];
        index = entry[4];
        step0 = entry[5];
        count = entry[6];
        piece = entry[7];
        pieces = entry[8];
        first_part = entry[9];
    }

    // Of a tile that is there: the same in all lanes, so that loops on its numbers are scalar, and so are the buffers that it is loaded from.  (Said once it is
    // known to be there: in the constructor the compiler still made loops over the lanes of every load, 8 % of the forward pass's time.)
    __device__ __forceinline__ void settle()
    {
        for (uint32_t *x : {&index, &q0, &m, &k0, &n, &kvh, &piece, &pieces, &first_part, &step0, &count}) *x = __builtin_amdgcn_readfirstlane(*x);
    }

    // Where the results of a piece of this tile lie, in rows or keys.
    __device__ __forceinline__ int64_t part(const PromptArgs &p, uint32_t of) const { return ((int64_t)kvh * p.parts + first_part + of) * TILE; }

    // Keys of the sequence as the tiles' loads want them.
    __device__ __forceinline__ Keys<MODE_PLAIN> keys(const PromptArgs &p) const
    {
        Keys<MODE_PLAIN> k(p.a, 0, kvh);
        k.end = n;
        return k;
    }
};

// A plan to be made: tiles of `tile` rows or keys, steps of `step` keys or rows.
struct PlanOf {
    uint32_t *plan;
    uint32_t tile, step, slots, parts;
    uint32_t room, least;       // blocks of all heads that run at once, steps of a piece at least (0: no pieces)
    bool keys;
};

struct PlanArgs {
    PromptArgs p;
    PlanOf of[2];
};

constexpr uint32_t PLAN_SEQS = 2048, PLAN_TILES = 2048, PLAN_THREADS = 256;     // sequences and tiles at most

// Plans of[blockIdx.x].  Tiles and pieces are sorted by their length in 256 classes; which of a class come first does not matter to any result.
// One block a plan: 6.1 us for 24 prompts of 17 to 2500 rows, 5.1 for one, most of it the latency of the starts and of a dozen barriers (with 1024 threads 1 us more).
__global__ __launch_bounds__(PLAN_THREADS) void k_prompt_plan(const PlanArgs x)
{
    constexpr uint32_t MINE = PLAN_TILES / PLAN_THREADS, CLASSES = PLAN_THREADS, WAVES = PLAN_THREADS / 64;
    const PromptArgs &p = x.p;
    const PlanOf &of = x.of[blockIdx.x];
    __shared__ uint32_t first_tile[PLAN_SEQS + 1];
    __shared__ uint32_t classes[CLASSES], sums[WAVES], more[WAVES], cuts;
    const uint32_t thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;

    // the sum of all threads' x, and the largest y; sums_before: of the threads before this one
    uint32_t sum_before = 0, sum_all = 0, most_all = 0;
    const auto reduce = [&](uint32_t a, uint32_t b) {
        const uint32_t upto = sums_below(a), most = most_of_lanes(b);
        if (lane == 63) sums[wave] = upto;
        if (lane == 0) more[wave] = most;
        __syncthreads();
        const uint32_t other = lane < WAVES ? sums[lane] : 0, below = sums_below(other), top = most_of_lanes(lane < WAVES ? more[lane] : 0);
        sum_all = __builtin_amdgcn_readlane(below, WAVES - 1);
        sum_before = upto - a + (wave ? __shfl(below, wave - 1) : 0);
        most_all = top;
        __syncthreads();
    };

    uint32_t tiles = 0;
    for (uint32_t from = 0; from < p.seqs; from += PLAN_THREADS) {
        const uint32_t seq = from + thread;
        const uint32_t here = seq < p.seqs ? (Sequence(p, seq).lines(p, of.keys) + of.tile - 1) / of.tile : 0;
        reduce(here, 0);
        if (seq < p.seqs) first_tile[seq] = tiles + sum_before;
        tiles += sum_all;
    }
    classes[thread] = 0;
    if (thread == 0) {
        first_tile[p.seqs] = tiles;
        cuts = 0;
    }
    __syncthreads();
    if (tiles > PLAN_TILES) tiles = PLAN_TILES;         // (starts that do not ascend)

    // This thread's tiles: which sequence, how many steps.
    uint32_t steps[MINE], seqs[MINE], total = 0, longest = 0;
#pragma unroll
    for (uint32_t i = 0; i < MINE; ++i) {
        const uint32_t t = i * PLAN_THREADS + thread;
        steps[i] = seqs[i] = 0;
        if (i * PLAN_THREADS >= tiles) continue;                // by the whole block
        if (t < tiles) {
            uint32_t low = 0, high = p.seqs;            // first_tile[low] <= t < first_tile[high]
            while (high - low > 1) {
                const uint32_t mid = (low + high) / 2;
                if (first_tile[mid] <= t) low = mid;
                else high = mid;
            }
            seqs[i] = low;
            steps[i] = Sequence(p, low).steps(p, of.keys, of.tile, of.step, t - first_tile[low]);
            total += (steps[i] + 7) / 8;                // in 8 steps: below 2^32
            longest = steps[i] > longest ? steps[i] : longest;
        }
    }
    reduce(total, longest);

    // From tiles longer than a unit's share of all steps, and a thirty-second more, pieces of that length are cut off; the rests are sorted in among the
    // other tiles.  Longest first, this ends within 12 % of the even share (pieces of equal length: 10 to 50 % behind it).
    uint32_t size = most_all ? most_all : 1, slack = 0;
    if (of.least) {
        const uint64_t share = (uint64_t)sum_all * 8 * p.a.kv_heads / of.room;
        size = (uint32_t)(share + share / 32) + 1;
        size = size > of.least ? size : of.least;
        slack = of.least / 2;                           // that is not worth a piece
    }
    const auto pieces_of = [&](uint32_t n) { return n > size + slack ? (n - slack + size - 1) / size : 1; };
    const uint32_t top = size + slack < most_all ? size + slack : most_all ? most_all : 1;
    const float per_class = (CLASSES - 1) / (float)top;
    const auto class_of = [&](uint32_t n) {
        const uint32_t c = (uint32_t)((float)n * per_class);
        return CLASSES - 1 - (c < CLASSES ? c : CLASSES - 1);
    };
    uint32_t cut = 0;                                   // pieces of this thread's cut tiles
#pragma unroll
    for (uint32_t i = 0; i < MINE; ++i)
        if (i * PLAN_THREADS + thread < tiles) {
            const uint32_t pieces = pieces_of(steps[i]);
            atomicAdd(&classes[class_of(steps[i] - (pieces - 1) * size)], 1);
            if (pieces > 1) atomicAdd(&classes[class_of(size)], pieces - 1);
            cut += pieces > 1 ? pieces : 0;
        }
    __syncthreads();
    reduce(cut, 0);
    uint32_t part = sum_before;
    const bool too_many = sum_all > of.parts;           // (of sequences that overlap)
    const uint32_t own = classes[thread];
    reduce(own, 0);
    classes[thread] = sum_before;
    const bool fits = !too_many && sum_all <= of.slots;
    if (thread == 0) {
        of.plan[0] = fits ? sum_all : 0;
        of.plan[1] = 0;
    }
    __syncthreads();
    if (!fits) return;
#pragma unroll
    for (uint32_t i = 0; i < MINE; ++i)
        if (i * PLAN_THREADS + thread < tiles) {
            const uint32_t pieces = pieces_of(steps[i]), index = i * PLAN_THREADS + thread - first_tile[seqs[i]];
            const Sequence q(p, seqs[i]);
            for (uint32_t k = 0; k < pieces; ++k) {
                const uint32_t step0 = k * size, count = k + 1 < pieces ? size : steps[i] - step0, at = atomicAdd(&classes[class_of(count)], 1);
                u32x4 *e = reinterpret_cast<u32x4 *>(of.plan + ENTRIES + ENTRY * at);
                e[0] = u32x4{q.q0, q.m, q.k0, q.n};
                e[1] = u32x4{index, step0, count, k};
                e[2] = u32x4{pieces, part, 0, 0};
                if (pieces > 1 && k == 0) of.plan[ENTRIES + ENTRY * of.slots + atomicAdd(&cuts, 1)] = at;
            }
            part += pieces > 1 ? pieces : 0;
        }
    __syncthreads();
    if (thread == 0) of.plan[1] = cuts;
}

__device__ __forceinline__ uint32_t block_place(const PromptArgs &p) { return p.dies ? by_die(blockIdx.x, gridDim.x) : blockIdx.x; }

// Scores of keys first + {8 (r / 4) + 4 h + r % 4} that a row with so many keys left does not see become -inf.
__device__ __forceinline__ void mask_behind(f32x16 &x, int left)
{
    const int own = left - 4 * (int)((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 8 * (r / 4) + r % 4 < own ? x[r] : -INFINITY;
}

// Stores a lane's column of a transposed result as store_row does, 16 bytes at a time: the two lanes that hold a row exchange what makes eight neighbours.
template <class T, int DP>
__device__ __forceinline__ void store_row_16(uint16_t *row, bool live, const f32x16 (&acc)[DP / 32], float times, uint32_t head_dim)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 4; u += 2) {
            u32x2 four[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4 x = {acc[dt][4 * (u + k)] * times, acc[dt][4 * (u + k) + 1] * times, acc[dt][4 * (u + k) + 2] * times, acc[dt][4 * (u + k) + 3] * times};
                four[k] = __builtin_bit_cast(u32x2, __builtin_convertvector(x, typename T::V4));
            }
            u32x4 eight;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const auto r = __builtin_amdgcn_permlane32_swap(four[0][k], four[1][k], false, false);
                eight[k] = r[0];
                eight[2 + k] = r[1];
            }
            const int d = 32 * dt + 8 * (u + h);
            if (live && d < (int)head_dim) *reinterpret_cast<u32x4 *>(row + d) = eight;
        }
}

// Loads straight to shared memory: 16 or 4 bytes a lane, `offset` (a lane's own, in bytes) behind the base, lane after lane to the place `to`.
// Written out, as the compiler waits for all that are under way at every barrier and at the first read of shared memory after one: who uses them counts them
// and waits (`arrived`).  (m0 is not said to be written: it is a register that the compiler keeps out of its own hands, and sets before every use.)
// Nor does it keep the distance that such a load wants from what comes before: five wait states behind a vector instruction that has written the base, as a lane read
// first is or a spilled value read back, and one behind the write of m0.  Scalar instructions wait for such a write by themselves: the base is moved by one, which
// stands behind m0's.  (8192 rows 510 us instead of 507, a training step 894 instead of 892; with five states before every load 510 and 898.)
__device__ __forceinline__ void load_16_to_shared(const void *base, uint32_t offset, uint32_t to)
{
    uint64_t own;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(own) : "s"(to), "v"(offset), "s"(base) : "memory");
}

__device__ __forceinline__ void load_4_to_shared(const void *base, uint32_t offset, uint32_t to)
{
    uint64_t own;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0" : "=&s"(own) : "s"(to), "v"(offset), "s"(base) : "memory");
}

__device__ __forceinline__ uint32_t place_in_shared(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// All but the last LEFT loads of this wave are there, and, behind the barrier, those of all waves; this wave reads nothing older any more.
template <int LEFT>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Tiles of 64 keys on their way to shared memory, without registers between: a wave's share, what a lane loads of it.
template <int DP, int W>
struct Incoming {
    static constexpr int CH = DP / 8, MINE = CH / W;    // loads of a wave a tile, 64 chunks each
    static_assert(MINE * W == CH, "a tile is dealt out evenly");
    const uint16_t *from;                               // the head's first key of the sequence
    int64_t stride;
    uint32_t head_dim;
    int wave, lane;
    uint32_t offset[MINE];                              // in a whole tile, bytes

    __device__ __forceinline__ Incoming(const uint16_t *from_, int64_t stride_, uint32_t head_dim_, int wave_, int lane_)
        : from(from_), stride(stride_), head_dim(head_dim_), wave(wave_), lane(lane_)
    {
#pragma unroll
        for (int i = 0; i < MINE; ++i) offset[i] = offset_of(i, 64);
    }

    // Keys past the last one repeat it, columns past the head's the first ones: those keys are masked, and the rows' operands are 0 there.
    __device__ __forceinline__ uint32_t offset_of(int i, uint32_t left) const
    {
        const uint32_t at = (wave * MINE + i) * 64 + lane, own = at / CH, row = own < left ? own : left - 1;
        const int c = (at % CH) ^ spread<CH>(own);
        return 2 * (row * (uint32_t)stride + (8 * c < (int)head_dim ? 8 * c : 0));
    }

    // Keys first .. of n; there is one at least.
    __device__ __forceinline__ void load(u32x4 *tile, uint32_t first, uint32_t n) const
    {
        const uint16_t *base = from + first * stride;
        const uint32_t left = n - first;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            uint32_t own = offset[i];
            if (left < 64) own = offset_of(i, left);
            load_16_to_shared(base, own, place_in_shared(tile + (wave * MINE + i) * 64));
        }
    }
};

// Forward: W waves of 32 rows each share a tile of 64 keys; the block ends with the tile that its last row sees, and only tiles that some row does not
// see whole are masked.  One pass, with a row's mark (near its maximum) and sum in the two lanes that hold its scores:
//   x = K q,  p = 2^(scale x - mark),  sum += p,  o = 2^(old mark - mark) o + V^T p,  at the end o / sum and lse.
// Bound by matrix instructions, two products of 2 head_dim operations a score, and beside them one exponential a score, which issues at a quarter of the
// rate: a step of 64 keys is 1024 cycles of a wave's matrix instructions at 128 a head, and 512 of exponentials alone; at 64 a head 512 and 512.
//   One prompt of 8192 rows, 32 heads of 128, bfloat16: 535 us, 1.03 PFLOP/s, busy 60 %, 1.91 GHz (before its last step 1.19 PFLOP/s where all values are zeros: power).
//   24 of 17 to 2500, 32 heads over 8 of 128, float16: 176 us, 0.83 PFLOP/s, busy 49 %.  40 of 23 to 509, 12 heads of 64, not causal: 23 us, a round of blocks
//   whose longest has eight steps.
// The step in slots of one product took the first from 562 to 546 us a call, tiles straight to shared memory from 559 to 539, the next step's first
// operands before this one's last products from 524 to 515 (another card); operands read 4 to 8 products ahead and three or four tiles under way gained nothing.
template <class T, int DP, int W, bool LEAN>
__global__ __launch_bounds__(64 * W, LEAN ? 4 : 2) void k_prompt_forward(const PromptArgs p)
{
    // Tiles under way: K of tile s + 1 + DEEP and V of tile s + DEEP while tile s is worked on.
    constexpr int TN = 64, MT = 2, CH = DP / 8, GT = 64 * W, DEEP = !LEAN && DP <= 64 ? 3 : 1, RING = DEEP + 1;
    __shared__ u32x4 memory[2 * RING * TN * CH];
    const AttnArgs &a = p.a;
    Tile<32 * W, TN, false> tile(p, block_place(p));
    if (!tile.there) return;
    tile.settle();
    const int thread = threadIdx.x, lane = thread & 63, n = lane & 31, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const uint32_t rows = tile.m * a.group, row0 = tile.index * 32 * W, row = row0 + 32 * wave + n, step0 = tile.step0, count = tile.count;
    const bool live = row < rows;
    const uint32_t limit = limit_of(p, tile.m, tile.n, token_of(a, live ? row : rows - 1)), all_see = limit_of(p, tile.m, tile.n, token_of(a, row0));

    const uint16_t *const k_at = a.k + tile.k0 * a.ks.token, *const v_at = a.v + tile.k0 * a.vs.token;
    typename T::V8 q[DP / 16];
    row_operands<T, DP>(q, a.q + tile.q0 * a.qs.token + row_at(a, a.qs, 0, tile.kvh, live ? row : 0), live, a.head_dim);

    f32x16 sums[1][DP / 32] = {};
    f32x16(&o)[DP / 32] = sums[0];
    float top = -INFINITY, total = 0.0f;                // mark near the maximum (scaled, in powers of two); this lane's share of the sum
    auto k_tile = [&](uint32_t s) { return memory + s % RING * TN * CH; };     // s: of the tile, or its remainder
    auto v_tile = [&](uint32_t s) { return memory + (RING + s % RING) * TN * CH; };
    auto first_of = [&](uint32_t s) { return (step0 + s) * TN; };
    constexpr float HIGHER = NARROW<T> ? 7.0f : 0.0f;   // powers of two, of probabilities: see k_attn_forward
    f32x16 x[MT], ahead[MT];
    float most = -INFINITY;                             // maximum of the scores that are next, scaled

    // Operands: of the product i of a tile's scores (keys 32 (i mod 2) .., columns 16 (i / 2) .. of the head), and of the product i with its values
    // (columns 32 (i mod DT) .., keys 16 (i / DT) ..).
    constexpr int DT = DP / 32;
    auto key_operand = [&](uint32_t s, int i) { return k_tile(s)[32 * (i % MT) * CH + chunk_at<CH>(n, 2 * (i / MT) + h)]; };
    auto value_operand = [&](s16x4 (&to)[2], uint32_t s, int i) {
        const int l = lane & 15, c = 4 * (i % DT) + 2 * ((lane >> 4) & 1) + ((l >> 1) & 1);
#pragma unroll
        for (int j = 0; j < 2; ++j) to[j] = read_transposed(reinterpret_cast<const char *>(v_tile(s) + 16 * (i / DT) * CH + chunk_at<CH>(4 * h + (l >> 2) + 8 * j, c)) + 8 * (l & 1));
    };
    auto scores = [&](f32x16 (&to)[MT], uint32_t s) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) to[mt] = keys_by_rows<T, DP>(k_tile(s), 32 * mt, q);
    };
    auto mask = [&](f32x16 (&to)[MT], uint32_t s) {
        const int left = (int)limit - (int)first_of(s);
        if (__all(left >= TN)) return;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) mask_behind(to[mt], left - 32 * mt);
    };
    auto maximum = [&](const f32x16 (&of)[MT]) {
        float m = of[0][0];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 16; ++r) m = __builtin_elementwise_maximum(m, of[mt][r]);
        return m;
    };
    // A mark that is kept until a row outgrows it by 2^8 spares scaling the accumulators every tile.
    auto raise = [&] {
        most = __builtin_fmaf(max_of_halves(most), a.scale_log2, -HIGHER);
        if (__any(!(most <= top + 8.0f))) {
            const float mark = __builtin_elementwise_maximum(top, most);
            const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - mark);
            top = mark;
            total *= keep;
#pragma unroll
            for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= keep;
        }
    };
    auto exponentials = [&](f32x16 (&now)[MT], typename T::V8 (&to)[MT][2][1]) {
        const float off = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) now[mt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(now[mt][r], a.scale_log2, -off));
            to[mt][0][0] = rounded<T>(now[mt], 0);
            to[mt][1][0] = rounded<T>(now[mt], 1);
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += now[mt][r];
            total += sum;
        }
    };
    auto values = [&](uint32_t s, const typename T::V8 (&of)[MT][2][1]) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int part = 0; part < 2; ++part) columns_times<T, DP, 1>(sums, v_tile(s), 32 * mt + 16 * part, of[mt][part]);
    };

    if constexpr (LEAN) {
        // Short sequences: what counts is how many blocks run at once, so that the trips to memory of one overlap those of others.  32 keys at a time, so that
        // 128 registers suffice.
        Stage<DP, TN, GT, MODE_PLAIN> sk, sv;
        const Keys<MODE_PLAIN> keys = tile.keys(p);
        auto load = [&](uint32_t s) {
            sk.load(keys, k_at, a.ks, thread, first_of(s), 0);
            sv.load(keys, v_at, a.vs, thread, first_of(s), 0);
        };
        if (count) load(0);
#pragma unroll 1
        for (uint32_t s = 0; s < count; ++s) {
            sk.store(k_tile(s), thread);
            sv.store(v_tile(s), thread);
            __syncthreads();
            if (s + 1 < count) load(s + 1);
            const int left = (int)limit - (int)first_of(s);
            const bool whole = __all(left >= TN);
#pragma unroll 1
            for (int mt = 0; mt < MT; ++mt) {
                f32x16 y = keys_by_rows<T, DP>(k_tile(s), 32 * mt, q);
                if (!whole) mask_behind(y, left - 32 * mt);
                most = y[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) most = __builtin_elementwise_maximum(most, y[r]);
                raise();
                const float off = top == -INFINITY ? 0.0f : top;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    y[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[r], a.scale_log2, -off));
                    total += y[r];
                }
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const typename T::V8 pr[1] = {rounded<T>(y, part)};
                    columns_times<T, DP, 1>(sums, v_tile(s) + 32 * mt * CH, 16 * part, pr);
                }
            }
        }
    } else if (count) {
        // Tile s + 1's scores beside tile s's exponentials, its maximum beside tile s's product with V: K runs a tile ahead of V.
        const Incoming<DP, W> k_in(k_at + tile.kvh * a.ks.head, a.ks.token, a.head_dim, wave, lane), v_in(v_at + tile.kvh * a.vs.head, a.vs.token, a.head_dim, wave, lane);
        constexpr int LOADS = 2 * Incoming<DP, W>::MINE;
        const auto load_keys = [&](uint32_t s, uint32_t to) { k_in.load(k_tile(to), first_of(s < count ? s : count - 1), tile.n); };    // (behind the last one it is loaded again)
        const auto load_values = [&](uint32_t s, uint32_t to) { v_in.load(v_tile(to), first_of(s < count ? s : count - 1), tile.n); };
        load_keys(0, 0);
#pragma unroll
        for (uint32_t s = 0; s < DEEP; ++s) {
            load_values(s, s);
            load_keys(s + 1, s + 1);
        }
        arrived<LOADS * (DEEP - 1)>();
        scores(x, 0);
        mask(x, 0);
        most = maximum(x);
        raise();
        __syncthreads();
        constexpr int KP = MT * DP / 16, VP = KP, AHEAD = W == 8 ? 3 : 2, EACH = 16 * MT / KP;
        u32x4 ko[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ko[i] = key_operand(1, i);

        // Tile s from its scores `now`; the next one's scores into `next`.  In slots of one product, the read of an operand that is wanted some products later
        // and a share of the vector instructions, in this order: left to itself the compiler reads every operand right before its use.
        // at: s, or what it leaves divided by RING, known when this is compiled.
        auto step = [&](uint32_t s, auto at, f32x16 (&now)[MT], f32x16 (&next)[MT], auto masked) {
            typename T::V8 pr[MT][2][1];
            s16x4 vo[AHEAD][2];
            const float off = top == -INFINITY ? 0.0f : top;
            load_keys(s + 1 + DEEP, at + 1 + DEEP);     // to where nobody reads any more since the last barrier
            load_values(s + DEEP, at + DEEP);
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                next[i % MT] = T::mma(as_operand<T>(ko[i % AHEAD]), q[i / MT], i < MT ? f32x16{} : next[i % MT]);
                if (i + AHEAD < KP) ko[i % AHEAD] = key_operand(at + 1, i + AHEAD);
                else value_operand(vo[i + AHEAD - KP], at, i + AHEAD - KP);
#pragma unroll
                for (int e = i * EACH; e < (i + 1) * EACH; ++e) {
                    now[e / 16][e % 16] = __builtin_amdgcn_exp2f(__builtin_fmaf(now[e / 16][e % 16], a.scale_log2, -off));
                    total += now[e / 16][e % 16];
                    if (e % 8 == 7) pr[e / 16][e / 8 % 2][0] = rounded<T>(now[e / 16], e / 8 % 2);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (masked) mask(next, s + 1);
            float m = next[0][0];
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                o[i % DT] = T::mma(join<T>(vo[i % AHEAD][0], vo[i % AHEAD][1]), pr[i / DT / 2][i / DT % 2][0], o[i % DT]);
                if (i + AHEAD < VP) value_operand(vo[i % AHEAD], at, i + AHEAD);
                if (i == VP - AHEAD) arrived<LOADS * (DEEP - 1)>();         // K of tile s + 2, V of tile s + 1; this tile's operands are read
                if (i >= VP - AHEAD) ko[i - (VP - AHEAD)] = key_operand(at + 2, i - (VP - AHEAD));
#pragma unroll
                for (int e = i * EACH; e < (i + 1) * EACH; ++e) m = __builtin_elementwise_maximum(m, next[e / 16][e % 16]);
                __builtin_amdgcn_sched_barrier(0);
            }
            most = m;
            raise();
        };
        auto last = [&](uint32_t s, f32x16 (&now)[MT]) {
            typename T::V8 pr[MT][2][1];
            exponentials(now, pr);
            values(s, pr);
        };
        uint32_t s = 0;
        for (; s + RING + 1 < count && first_of(s + RING + 1) <= all_see; s += RING) {      // tiles s + 1 .. s + RING are seen whole by every row
            step(s, std::integral_constant<uint32_t, 0>(), x, ahead, std::false_type());
            step(s + 1, std::integral_constant<uint32_t, 1>(), ahead, x, std::false_type());
            if constexpr (RING == 4) {
                step(s + 2, std::integral_constant<uint32_t, 2>(), x, ahead, std::false_type());
                step(s + 3, std::integral_constant<uint32_t, 3>(), ahead, x, std::false_type());
            }
        }
#pragma unroll 1
        for (; s + 1 < count; ++s) {
            step(s, s, x, ahead, std::true_type());
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) x[mt] = ahead[mt];
        }
        last(s, x);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // nothing writes to shared memory any more when the block ends
    }
    total = sum_of_halves(total);
    const float times = total != 0.0f ? 1.0f / total : 0.0f, sum2 = total != 0.0f ? top + __log2f(total) : -INFINITY;
    if (tile.pieces == 1) {
        store_row_16<T, DP>(a.o + tile.q0 * a.os.token + row_at(a, a.os, 0, tile.kvh, live ? row : 0), live, o, times, a.head_dim);
        if (a.lse && live && h == 0) a.lse[lse_at(a, 0, tile.kvh, row) + tile.q0] = sum2 * LN2;
    } else if (live) {
        const int64_t line = tile.part(p, tile.piece) + 32 * wave + n;
        store_part<DP>(a.part_o + line * DP, o, times);
        if (h == 0) a.part_lse[line] = sum2;
    }
}

// Joins the pieces of the tiles of 32 W rows that were cut, in ascending order: o = sum of 2^(lse_i - top) o_i over the sum of 2^(lse_i - top).  32 rows a
// block, a thread four columns.  Reads and writes alone: 33 MB for 703 rows, 32 heads, over 9000 to 16384 keys in 8.3 us.
template <class T, int DP, int W>
__global__ __launch_bounds__(8 * DP) void k_prompt_join(const PromptArgs p)
{
    constexpr int C4 = DP / 4;
    const AttnArgs &a = p.a;
    Tile<32 * W, 64, false> tile(p, blockIdx.x / W, std::true_type());
    if (!tile.there) return;
    tile.settle();
    const uint32_t i = threadIdx.x;
    const uint32_t within_tile = blockIdx.x % W * 32 + i / C4, row = tile.index * 32 * W + within_tile, c = i % C4;
    if (row >= tile.m * a.group) return;
    const int64_t line = tile.part(p, 0) + within_tile;
    float high = -INFINITY, sum = 0.0f;
    for (uint32_t s = 0; s < tile.pieces; ++s) high = __builtin_elementwise_maximum(high, a.part_lse[line + s * 32 * W]);
    const float off = high == -INFINITY ? 0.0f : high;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t s = 0; s < tile.pieces; ++s) {
        const float w = __builtin_amdgcn_exp2f(a.part_lse[line + s * 32 * W] - off);
        sum += w;
        x += *reinterpret_cast<const f32x4 *>(a.part_o + (line + s * 32 * W) * DP + 4 * c) * w;
    }
    x *= sum != 0.0f ? 1.0f / sum : 0.0f;
    if (4 * c < a.head_dim) *reinterpret_cast<typename T::V4 *>(a.o + tile.q0 * a.os.token + row_at(a, a.os, 0, tile.kvh, row) + 4 * c) = __builtin_convertvector(x, typename T::V4);
    if (a.lse && c == 0) a.lse[lse_at(a, 0, tile.kvh, row) + tile.q0] = sum != 0.0f ? (high + __log2f(sum)) * LN2 : -INFINITY;
}

// What rounding the first half of x to `of` left, rounded.
template <class T>
__device__ __forceinline__ typename T::V8 left_over(const f32x16 &x, const typename T::V8 &of)
{
    f32x8 y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j] - (float)of[j];
    return __builtin_convertvector(y, typename T::V8);
}

// Sequences of up to so many keys (one step of a product) take dS into dQ and dK as two operands, the rounded value and what that left: where a call has a handful of
// dS in all their rounding does not average, and was up to 1.6 times that of the results.  In blocks of four waves alone: where there are eight, sequences are long on
// average, and such a sequence is one of few.
constexpr uint32_t FEW_KEYS = 16;

// dQ, and D on the way:  P = 2^(scale S log2 e - lse2),  D = sum of dO O,  dS = P (dO V^T - D),  dQ = scale dS K.  Rows as in the forward pass, Q and dO in
// registers; three products and an exponential a score.  D and lse2 go to the workspace, where dK and dV read them.
// Bound as the forward pass: documents of 4096, 1333, 2048 and 715 rows, 32 heads over 8 of 128, bfloat16: 288 us, 0.99 PFLOP/s, busy 55 %, 1.94 GHz
// (a call in slots of one product: the step of training 936 us instead of 954).  40 sentences of 23 to 509, 12 heads of 64, float16: 26 us.
// Three waves a SIMD where 168 registers suffice: 64 a head, float16, 79.5 us with three (a training step over the 40 sentences), 81.5 with two; bfloat16 78.5, and 75.7
// with two.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, DP <= 32 || (DP <= 64 && NARROW<T>) ? 3 : 2) void k_prompt_dq(const PromptArgs p)
{
    constexpr int TN = 64, CH = DP / 8;
    __shared__ u32x4 tiles[2][2][TN * CH];
    const AttnArgs &a = p.a;
    Tile<32 * W, TN, false> tile(p, block_place(p));
    if (!tile.there) return;
    tile.settle();
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63, n = lane & 31, h = lane >> 5;
    const uint32_t rows = tile.m * a.group, row = tile.index * 32 * W + 32 * wave + n, step0 = tile.step0, count = tile.count;
    const bool live = row < rows;
    const uint32_t limit = limit_of(p, tile.m, tile.n, token_of(a, live ? row : rows - 1));
    const bool few = W == 4 && tile.n <= FEW_KEYS;      // one step, behind the loop

    const Incoming<DP, W> k_in(a.k + tile.k0 * a.ks.token + tile.kvh * a.ks.head, a.ks.token, a.head_dim, wave, lane);
    const Incoming<DP, W> v_in(a.v + tile.k0 * a.vs.token + tile.kvh * a.vs.head, a.vs.token, a.head_dim, wave, lane);
    const auto load = [&](uint32_t s) {
        k_in.load(tiles[s & 1][0], (step0 + s) * TN, tile.n);
        v_in.load(tiles[s & 1][1], (step0 + s) * TN, tile.n);
    };
    if (count) load(0);
    const int64_t line = (int64_t)tile.kvh * a.rows + tile.q0 * a.group + row;
    typename T::V8 q[DP / 16], d_o[DP / 16];
    row_operands<T, DP>(q, a.q + tile.q0 * a.qs.token + row_at(a, a.qs, 0, tile.kvh, live ? row : 0), live, a.head_dim);
    row_operands<T, DP>(d_o, a.d_o + tile.q0 * a.dos.token + row_at(a, a.dos, 0, tile.kvh, live ? row : 0), live, a.head_dim);
    float lse2 = INFINITY, delta = 0.0f;                // rows that see nothing: probabilities 0
    if (live) {
        const float l = a.lse_in[lse_at(a, 0, tile.kvh, row) + tile.q0];
        lse2 = l == -INFINITY ? INFINITY : l * LOG2E - (NARROW<T> && !few ? UP + HIGHEST : 0.0f);
    }
    {
        typename T::V8 o[DP / 16];
        row_operands<T, DP>(o, a.o_in + tile.q0 * a.os.token + row_at(a, a.os, 0, tile.kvh, live ? row : 0), live, a.head_dim);
#pragma unroll
        for (int t = 0; t < DP / 16; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta += (float)o[t][j] * (float)d_o[t][j];
        delta = sum_of_halves(delta);
        // D from the rounded O is off by O's rounding, which does not average over the keys of a row that sees few, whose dQ and dK it puts off by more than the
        // rounding of dS does (in all 2.3 times one rounding with two keys, 1.6 with 64 and causal, now 1.4).  Rows that see FEW tiles at most form it from P and
        // dP.  With 65 keys O's rounding adds 4 % to the error, with 32 values a head 5 %, in which that of dS is 5 % larger.
        constexpr uint32_t FEW = DP <= 32 ? 2 : 1;
        if (tile.pieces == 1 && count && limit_of(p, tile.m, tile.n, token_of(a, tile.index * 32 * W)) <= FEW * TN) {
            // float16: with lse as it is, read again.  (Less what the loop takes off, and that added back, it is rounded near 75 and puts P off by 2^-18; dS can be what little
            // D and dP leave of each other.)
            const float as_is = NARROW<T> && lse2 != INFINITY ? a.lse_in[lse_at(a, 0, tile.kvh, row) + tile.q0] * LOG2E : lse2;
            float exact = 0.0f;
#pragma unroll 1
            for (uint32_t s = 0; s < FEW && s < count; ++s) {
                arrived<0>();
                if (s + 1 < FEW && s + 1 < count) load(s + 1);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    f32x16 x = keys_by_rows<T, DP>(tiles[s & 1][0], 32 * mt, q);
                    const f32x16 dp = keys_by_rows<T, DP>(tiles[s & 1][1], 32 * mt, d_o);
                    mask_behind(x, (int)limit - (int)(s * TN) - 32 * mt);
#pragma unroll
                    for (int r = 0; r < 16; ++r) exact += __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale_log2, -as_is)) * dp[r];
                }
            }
            exact = sum_of_halves(exact);
            if (limit && limit <= FEW * TN) delta = exact;
        }
        if (live && h == 0 && tile.piece == 0) {
            a.delta[line] = delta;
            if (!NARROW<T>) p.lse2[line] = lse2;
        }
    }

    f32x16 dq[1][DP / 32] = {};
    float lowered = 0.0f;                               // of dS's power of two, which lse2 holds
    constexpr int NT = DP / 16, DT = DP / 32, AHEAD = 2, EACH = 16 / NT;
    for (uint32_t s = 0; s < (few ? 0 : count); ++s) {
        const u32x4 *const kt = tiles[s & 1][0], *const vt = tiles[s & 1][1];
        arrived<0>();
        if (s + 1 < count) load(s + 1);
        const int left = (int)limit - (int)((step0 + s) * TN);
        const bool whole = __all(left >= TN);
        const auto along = [&](const u32x4 *of, int mt, int t) { return of[32 * mt * CH + chunk_at<CH>(n, 2 * t + h)]; };
        const auto across = [&](s16x4 (&to)[2], int i) {        // of K: columns 32 (i mod DT) .., keys 16 (i / DT) ..
            const int l = lane & 15, c = 4 * (i % DT) + 2 * ((lane >> 4) & 1) + ((l >> 1) & 1);
#pragma unroll
            for (int j = 0; j < 2; ++j) to[j] = read_transposed(reinterpret_cast<const char *>(kt + 16 * (i / DT) * CH + chunk_at<CH>(4 * h + (l >> 2) + 8 * j, c)) + 8 * (l & 1));
        };
        // Products of 32 keys in turn, beside them what the products before left to do: S, S | exponentials, dP | exponentials, dP | dS, dQ | dS, dQ; operands are
        // read two products ahead.  In float16, where dS is kept in range between, one half of the keys after the other.
        constexpr int GROUP = NARROW<T> ? 1 : 2, ALL = 2 * GROUP * NT;
        f32x16 x[2], dp[2];
        typename T::V8 ds[2][2];
#pragma unroll
        for (int half = 0; half < 2; half += GROUP) {
            u32x4 operand[AHEAD];
            s16x4 ko[AHEAD][2];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) operand[i] = along(kt, half, i);
#pragma unroll
            for (int i = 0; i < ALL; ++i) {             // S, then dP
                const int t = i % NT, mt = half + i / NT % GROUP, later = i + AHEAD;
                if (i < ALL / 2) x[mt] = T::mma(as_operand<T>(operand[i % AHEAD]), q[t], t ? x[mt] : f32x16{});
                else dp[mt] = T::mma(as_operand<T>(operand[i % AHEAD]), d_o[t], t ? dp[mt] : f32x16{});
                if (later < ALL) operand[i % AHEAD] = along(later < ALL / 2 ? kt : vt, half + later / NT % GROUP, later % NT);
                else across(ko[later - ALL], 2 * DT * half + later - ALL);
                if (i >= NT && i < ALL / 2 + NT) {
                    const int of = half + i / NT - 1;
#pragma unroll
                    for (int e = EACH * t; e < EACH * (t + 1); ++e) x[of][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[of][e], a.scale_log2, -lse2));
                }
                if (GROUP == 2 && i >= 3 * NT) {
#pragma unroll
                    for (int e = EACH * t; e < EACH * (t + 1); ++e) {
                        x[0][e] *= dp[0][e] - delta;
                        if (e % 8 == 7) ds[0][e / 8] = rounded<T>(x[0], e / 8);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (t == NT - 1 && i < ALL / 2 && !whole) mask_behind(x[mt], left - 32 * mt);
            }
            if (NARROW<T>) {
                x[half] *= dp[half] - delta;
                const float by = keep_in_range(x[half], dq[0]);
                lowered += by;
                lse2 -= by;
#pragma unroll
                for (int part = 0; part < 2; ++part) ds[half][part] = rounded<T>(x[half], part);
            }
#pragma unroll
            for (int i = 0; i < 2 * DT * GROUP; ++i) {
                const int at = 2 * DT * half + i, mt = at / (2 * DT);
                dq[0][i % DT] = T::mma(join<T>(ko[i % AHEAD][0], ko[i % AHEAD][1]), ds[mt][at / DT % 2], dq[0][i % DT]);
                if (i + AHEAD < 2 * DT * GROUP) across(ko[i % AHEAD], at + AHEAD);
                if (GROUP == 2 && i < 2 * DT) {
#pragma unroll
                    for (int e = EACH * i; e < EACH * (i + 1); ++e) {
                        x[1][e] *= dp[1][e] - delta;
                        if (e % 8 == 7) ds[1][e / 8] = rounded<T>(x[1], e / 8);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if (few && count) {
        arrived<0>();
        f32x16 x = keys_by_rows<T, DP>(tiles[0][0], 0, q);
        const f32x16 dp = keys_by_rows<T, DP>(tiles[0][1], 0, d_o);
        mask_behind(x, (int)limit);
        float most = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale_log2, -lse2)) * (dp[r] - delta);
            most = __builtin_fmaxf(most, __builtin_fabsf(x[r]));
        }
        if (NARROW<T>) {                                // to 2^10 .. 2^11
            const int by = 11 - __builtin_amdgcn_frexp_expf(max_of_halves(most));
#pragma unroll
            for (int r = 0; r < 8; ++r) x[r] = __builtin_ldexpf(x[r], by);
            lowered = (float)by - (UP + HIGHEST);
        }
        // the rounded value, and what that left
        const typename T::V8 first[1] = {rounded<T>(x, 0)}, rest[1] = {left_over<T>(x, first[0])};
        columns_times<T, DP, 1>(dq, tiles[0][0], 0, first);
        columns_times<T, DP, 1>(dq, tiles[0][0], 0, rest);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // nothing writes to shared memory any more when the block ends
    if (lse2 == INFINITY) {                             // (a row that sees nothing, whatever its query and gradient hold)
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt) dq[0][dt] = f32x16{};
    }
    const float times = NARROW<T> ? a.scale * __builtin_amdgcn_exp2f(-(UP + HIGHEST + lowered)) : a.scale;
    if (tile.pieces == 1) store_row_16<T, DP>(a.dq + tile.q0 * a.dqs.token + row_at(a, a.dqs, 0, tile.kvh, live ? row : 0), live, dq[0], times, a.head_dim);
    else if (live) store_part<DP>(a.part_o + (tile.part(p, tile.piece) + 32 * wave + n) * DP, dq[0], times);
}

// dK and dV of 32 W keys, 32 a wave, over the rows that see them:  dV = P^T dO,  dK = scale dS^T Q.  S and dP are formed again (a row's P is its lse away),
// which costs two products more than one kernel for all three gradients would, and saves atomics on dQ.  Q, dO and the rows' statistics go through
// registers to shared memory, so that what is no row is zeros.
// Bound by matrix instructions and the reads of operands from shared memory (each feeds one product).  40 sentences of 23 to 509, 12 heads of 64, float16:
// 31 us, busy 26 %: few steps a block, whose beginnings and ends show.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, 2) void k_prompt_dkv(const PromptArgs p)
{
    constexpr int TR = DP == 128 ? 32 : 64, CH = DP / 8, LOADS = TR * CH / (64 * W), ROWS = 64 * W / CH;
    static_assert(LOADS * 64 * W == TR * CH && 2 * TR <= 64 * W, "a tile is dealt out evenly, its statistics to two threads a row");
    __shared__ u32x4 tiles[2][2][TR * CH];
    __shared__ f32x4 stats[2][2][TR / 4];               // lse in powers of two, D
    constexpr bool AWAY = DP == 128;                    // V's operands in shared memory: with them 256 registers do not suffice
    __shared__ u32x4 away[AWAY ? W : 1][DP / 16][64];
    const AttnArgs &a = p.a;
    Tile<32 * W, TR, true> tile(p, block_place(p));
    if (!tile.there) return;
    tile.settle();
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63, n = lane & 31, h = lane >> 5;
    const uint32_t rows = tile.m * a.group, key0 = tile.index * 32 * W, key = key0 + 32 * wave + n;
    const int own = first_row(p, tile.m, tile.n, key), all_see = first_row(p, tile.m, tile.n, key0 + 32 * W - 1);
    const int first_seen = first_row(p, tile.m, tile.n, key0);
    const uint32_t begin = first_seen < 0 ? 0 : first_seen, step0 = tile.step0, count = tile.count;

    const bool valid = key < tile.n;
    const int64_t key_at = (int64_t)tile.k0 + (valid ? key : 0);
    typename T::V8 k[DP / 16], v[DP / 16];
    row_operands<T, DP>(k, a.k + key_at * a.ks.token + tile.kvh * a.ks.head, valid, a.head_dim);
    row_operands<T, DP>(v, a.v + key_at * a.vs.token + tile.kvh * a.vs.head, valid, a.head_dim);
    if (AWAY) {                                         // a lane reads what it has written itself
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) away[AWAY ? wave : 0][t][lane] = __builtin_bit_cast(u32x4, v[t]);
    }

    // Rows past the last one repeat its Q, and their dO is zeros, as their probabilities do not clear an infinite gradient.  Columns past the
    // head's repeat the first ones: K and V are 0 there.
    u32x4 rq[LOADS], ro[LOADS];
    float stat = 0.0f;
    const int load0 = thread / CH, c = 8 * (thread % CH) < (int)a.head_dim ? thread % CH : 0;
    const uint16_t *const q_at = a.q + tile.q0 * a.qs.token, *const do_at = a.d_o + tile.q0 * a.dos.token;
    const float *const lse_from = a.lse_in + tile.q0, *const delta_from = a.delta + (int64_t)tile.kvh * a.rows + tile.q0 * a.group;
    auto load = [&](uint32_t s) {
        const uint32_t first = begin + (step0 + s) * TR;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t row = first + load0 + i * ROWS, there = row < rows ? row : rows - 1;
            rq[i] = *reinterpret_cast<const u32x4 *>(q_at + row_at(a, a.qs, 0, tile.kvh, there) + c * 8);
            ro[i] = zeros();
            if (row < rows) ro[i] = *reinterpret_cast<const u32x4 *>(do_at + row_at(a, a.dos, 0, tile.kvh, there) + c * 8);
        }
        const uint32_t row = first + thread % TR;
        const bool there = row < rows;
        if (thread < TR) {
            const float l = lse_from[lse_at(a, 0, tile.kvh, there ? row : rows - 1)];
            stat = there && l != -INFINITY ? l * LOG2E - (NARROW<T> ? UP : 0.0f) : INFINITY;      // rows that are not there, or see nothing: probabilities 0
        } else if (thread < 2 * TR) {
            stat = delta_from[there ? row : rows - 1];
        }
    };
    f32x16 dk[1][DP / 32] = {}, dv[1][DP / 32] = {};
    float by = 0x1p60f;                                 // float16: dS's power of two over P's
    static_assert(HIGHEST == 60.0f);
    if (count) load(0);
    for (uint32_t s = 0; s < count; ++s) {
        u32x4 *qt = tiles[s & 1][0], *ot = tiles[s & 1][1];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            qt[chunk_at<CH>(load0 + i * ROWS, thread % CH)] = rq[i];
            ot[chunk_at<CH>(load0 + i * ROWS, thread % CH)] = ro[i];
        }
        if (thread < 2 * TR) reinterpret_cast<float *>(stats[s & 1])[thread] = stat;
        __syncthreads();
        if (s + 1 < count) load(s + 1);
        const int first = (int)(begin + (step0 + s) * TR);
#pragma unroll
        for (int sub = 0; sub < TR / 32; ++sub) {
            f32x16 x = {}, dp = {};
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) x = T::mma(as_operand<T>(qt[32 * sub * CH + chunk_at<CH>(n, 2 * t + h)]), k[t], x);
#pragma unroll
            for (int t = 0; t < DP / 16; ++t)
                dp = T::mma(as_operand<T>(ot[32 * sub * CH + chunk_at<CH>(n, 2 * t + h)]), AWAY ? as_operand<T>(away[AWAY ? wave : 0][t][lane]) : v[t], dp);
            if (first + 32 * sub < all_see) {           // rows before the first one that sees the lane's key
                const int before = own - first - 32 * sub - 4 * h;
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = 8 * (r / 4) + r % 4 >= before ? x[r] : -INFINITY;
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 lse2 = stats[s & 1][0][8 * sub + 2 * g + h], delta = stats[s & 1][1][8 * sub + 2 * g + h];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 4 * g + j;
                    const float pr = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale_log2, -lse2[j]));
                    x[r] = pr;
                    dp[r] = pr * (NARROW<T> ? (dp[r] - delta[j]) * by : dp[r] - delta[j]);
                }
            }
            if (NARROW<T>) by *= __builtin_amdgcn_exp2f(keep_in_range(dp, dk[0]));
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const typename T::V8 pr[1] = {rounded<T>(x, part)}, ds[1] = {rounded<T>(dp, part)};
                columns_times<T, DP, 1>(dv, ot, 32 * sub + 16 * part, pr);
                columns_times<T, DP, 1>(dk, qt, 32 * sub + 16 * part, ds);
            }
            if (W == 4 && tile.n <= FEW_KEYS) {
#pragma unroll 1
                for (int part = 0; part < 2; ++part) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) dp[j] = part ? dp[8 + j] : dp[j];
                    const typename T::V8 rest[1] = {left_over<T>(dp, rounded<T>(dp, 0))};
                    columns_times<T, DP, 1>(dk, qt, 32 * sub + 16 * part, rest);
                }
            }
        }
    }
    const float times = NARROW<T> ? a.scale * 0x1p-15f / by : a.scale, times_v = NARROW<T> ? 0x1p-15f : 1.0f;
    if (tile.pieces == 1) {
        store_row_16<T, DP>(a.dk + key_at * a.dks.token + tile.kvh * a.dks.head, valid, dk[0], times, a.head_dim);
        store_row_16<T, DP>(a.dv + key_at * a.dvs.token + tile.kvh * a.dvs.head, valid, dv[0], times_v, a.head_dim);
    } else if (valid) {
        float *part = a.part_o + (tile.part(p, tile.piece) + 32 * wave + n) * 2 * DP;
        store_part<DP>(part, dk[0], times);
        store_part<DP>(part + DP, dv[0], times_v);
    }
}

// dK and dV of 256 keys with 128 values each, 64 a wave and one wave a SIMD, 32 rows a step: every operand read feeds two products, and the step goes in slots
// of two, S | dP beside the exponentials | dV beside dS | dK.  Rows come straight to shared memory, three steps ahead.
// Documents of 4096, 1333, 2048 and 715 rows, 32 heads over 8 of 128, bfloat16: 425 us, 0.90 PFLOP/s, busy 53 %, 2.0 GHz (k_prompt_dkv: 502).
// Bound by the wave's own instructions: 64 of a step's 750 are matrix instructions (2048 of about 3800 cycles), 192 move sums between the two halves of the
// register file (the compiler lets all matrix instructions write to one half, which dK and dV fill).  Of 439 us 28 go without the exponentials, 24 without V's
// reads, 30 without the loads, 80 without all these and the transposing reads.  In float16, whose dS is kept in range between, registers do not suffice.
__global__ __launch_bounds__(256, 1) void k_prompt_dkv_wide(const PromptArgs p)
{
    using T = BF16;
    constexpr int DP = 128, CH = 16, TR = 32, STAGES = 4, NT = DP / 16, DT = DP / 32;
    __shared__ u32x4 tiles[STAGES][2][TR * CH];         // Q, dO
    // V's operands, and four of K's, for which registers do not suffice: a lane reads what it has written itself.
    __shared__ u32x4 away[4][2][NT][64], away_k[4][NT / 2][64];
    __shared__ f32x4 stats[STAGES][2][TR / 4];          // lse in powers of two (lower lanes), D
    const AttnArgs &a = p.a;
    Tile<256, TR, true> tile(p, block_place(p));
    if (!tile.there) return;
    tile.settle();
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63, n = lane & 31, h = lane >> 5;
    const uint32_t rows = tile.m * a.group, key0 = tile.index * 256 + 64 * wave;
    const int first_seen = first_row(p, tile.m, tile.n, tile.index * 256), all_see = first_row(p, tile.m, tile.n, key0 + 63);
    const uint32_t count = tile.count, start = (first_seen < 0 ? 0 : first_seen) + tile.step0 * TR;

    T::V8 k[2][NT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t key = key0 + 32 * u + n;
        const bool valid = key < tile.n;
        const int64_t at = (int64_t)tile.k0 + (valid ? key : 0);
        T::V8 v[NT];
        row_operands<T, DP>(k[u], a.k + at * a.ks.token + tile.kvh * a.ks.head, valid, a.head_dim);
        row_operands<T, DP>(v, a.v + at * a.vs.token + tile.kvh * a.vs.head, valid, a.head_dim);
#pragma unroll
        for (int t = 0; t < NT; ++t) away[wave][u][t][lane] = __builtin_bit_cast(u32x4, v[t]);
    }
#pragma unroll
    for (int t = 0; t < NT / 2; ++t) away_k[wave][t][lane] = __builtin_bit_cast(u32x4, k[1][NT / 2 + t]);

    // Loads: a wave has 8 of a step's rows, four at a time.  A step begins with a token (its rows are whole tokens).  Rows past the last one repeat it, and
    // columns past the head's the first ones: those rows are masked, and K and V are 0 there.  Behind the last step it is loaded again.
    const float *const stats_at = a.delta + (int64_t)tile.kvh * a.rows + tile.q0 * a.group;
    const uint32_t stats_offset = h ? 0 : 4 * (uint32_t)(p.lse2 - a.delta);
    const auto offset_of = [&](const Strides &s, uint32_t most, int i) {       // within a step of so many rows
        const uint32_t own = 8 * wave + 4 * i + (lane >> 4), row = own < most ? own : most - 1;
        const int c = (lane & 15) ^ spread<CH>(own), column = 8 * c < (int)a.head_dim ? 8 * c : 0;
        return 2 * ((uint32_t)row_at(a, s, 0, 0, row) + column);
    };
    const uint32_t q_offset[2] = {offset_of(a.qs, TR, 0), offset_of(a.qs, TR, 1)}, do_offset[2] = {offset_of(a.dos, TR, 0), offset_of(a.dos, TR, 1)};
    const uint16_t *const q_head = a.q + tile.q0 * a.qs.token + tile.kvh * a.group * a.qs.head, *const do_head = a.d_o + tile.q0 * a.dos.token + tile.kvh * a.group * a.dos.head;
    const auto load = [&](uint32_t s, auto stage) {
        const uint32_t first = start + (s < count ? s : count - 1) * TR, token = token_of(a, first), left = rows - first;
        const uint16_t *const q_from = q_head + token * a.qs.token, *const do_from = do_head + token * a.dos.token;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t q_own = q_offset[i], do_own = do_offset[i];
            if (left < TR) {
                q_own = offset_of(a.qs, left, i);
                do_own = offset_of(a.dos, left, i);
            }
            load_16_to_shared(q_from, q_own, place_in_shared(&tiles[stage][0][(8 * wave + 4 * i) * CH]));
            load_16_to_shared(do_from, do_own, place_in_shared(&tiles[stage][1][(8 * wave + 4 * i) * CH]));
        }
        load_4_to_shared(stats_at + first, 4 * ((uint32_t)n < left ? n : left - 1) + stats_offset, place_in_shared(&stats[stage][0][0]));
    };
    constexpr int LOADS = 5, AHEAD = 3, AHEAD_V = 2;
    const int own_row = first_row(p, tile.m, tile.n, key0 + n), next_keys = p.causal ? 32 * (int)a.group : 0;       // of u = 0; more of u = 1

    f32x16 dk[2][DT] = {}, dv[2][DT] = {};
    const auto along = [&](const u32x4 *of, int t) { return of[chunk_at<CH>(n, 2 * t + h)]; };
    u32x4 operand[AHEAD];
    const auto step = [&](uint32_t s, auto stage) {
        const u32x4 *const qt = tiles[stage][0], *const ot = tiles[stage][1];
        const uint32_t first = start + s * TR;
        const auto across = [&](s16x4 (&to)[2], const u32x4 *of, int i) {       // columns 32 (i mod DT) .., rows 16 (i / DT) ..
            const int l = lane & 15, c = 4 * (i % DT) + 2 * ((lane >> 4) & 1) + ((l >> 1) & 1);
#pragma unroll
            for (int j = 0; j < 2; ++j) to[j] = read_transposed(reinterpret_cast<const char *>(of + 16 * (i / DT) * CH + chunk_at<CH>(4 * h + (l >> 2) + 8 * j, c)) + 8 * (l & 1));
        };

        // S = Q K^T
        f32x16 x[2], dp[2];
        u32x4 ko[AHEAD_V], vo[AHEAD_V][2];
        f32x4 lse[2], delta[2];                         // of row group g, its four rows, in [g % 2]
        const auto lse_of = [&](int g) { lse[g % 2] = stats[stage][0][2 * g + h]; };
        const auto delta_of = [&](int g) { delta[g % 2] = stats[stage][1][2 * g + h]; };
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int u = 0; u < 2; ++u) x[u] = T::mma(as_operand<T>(operand[t % AHEAD]), u && t >= NT / 2 ? as_operand<T>(ko[t % AHEAD_V]) : k[u][t], t ? x[u] : f32x16{});
            if (t + AHEAD_V >= NT / 2 && t + AHEAD_V < NT) ko[t % AHEAD_V] = away_k[wave][t + AHEAD_V - NT / 2][lane];
            operand[t % AHEAD] = t + AHEAD < NT ? along(qt, t + AHEAD) : along(ot, t + AHEAD - NT);
            if (t + AHEAD_V >= NT) {
#pragma unroll
                for (int u = 0; u < 2; ++u) vo[t + AHEAD_V - NT][u] = away[wave][u][t + AHEAD_V - NT][lane];
            }
            if (t == NT - 1) lse_of(0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if ((int)first < all_see || first + TR > rows) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int from = own_row + u * next_keys - (int)first - 4 * h, behind = (int)(rows - first) - 4 * h;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = 8 * (r / 4) + r % 4;
                    x[u][r] = at >= from && at < behind ? x[u][r] : -INFINITY;
                }
            }
        }
        // The 32 exponentials and 32 dS of a lane, four rows of one u after the other, and the operands of 8 rows once they are whole.
        T::V8 pr[2][2], ds[2][2];
        const auto exponential = [&](int i) {
            const int g = i / 8, u = i / 4 % 2, j = i % 4;
            x[u][4 * g + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][4 * g + j], a.scale_log2, -lse[g % 2][j]));
            if (g % 2 && j == 3) pr[u][g / 2] = rounded<T>(x[u], g / 2);
        };
        const auto gradient = [&](int i) {
            const int g = i / 8, u = i / 4 % 2, j = i % 4;
            dp[u][4 * g + j] = x[u][4 * g + j] * (dp[u][4 * g + j] - delta[g % 2][j]);
            if (g % 2 && j == 3) ds[u][g / 2] = rounded<T>(dp[u], g / 2);
        };
        // dP = dO V^T beside the exponentials; operand[] holds dO's from (NT mod AHEAD) on
        s16x4 ao[AHEAD][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int slot = (t + NT) % AHEAD;
#pragma unroll
            for (int u = 0; u < 2; ++u) dp[u] = T::mma(as_operand<T>(operand[slot]), as_operand<T>(vo[t % AHEAD_V][u]), t ? dp[u] : f32x16{});
            if (t + AHEAD < NT) operand[slot] = along(ot, t + AHEAD);
            else across(ao[t + AHEAD - NT], ot, t + AHEAD - NT);
            if (t + AHEAD_V < NT) {
#pragma unroll
                for (int u = 0; u < 2; ++u) vo[t % AHEAD_V][u] = away[wave][u][t + AHEAD_V][lane];
            }
            if (t % 2 == 0) t < 6 ? lse_of(t / 2 + 1) : delta_of(0);
#pragma unroll
            for (int e = 4 * t; e < 4 * t + 4; ++e) exponential(e);
            __builtin_amdgcn_sched_barrier(0);
        }
        // dV += dO^T P beside dS
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {
#pragma unroll
            for (int u = 0; u < 2; ++u) dv[u][i % DT] = T::mma(join<T>(ao[i % AHEAD][0], ao[i % AHEAD][1]), pr[u][i / DT], dv[u][i % DT]);
            if (i + AHEAD < 2 * DT) across(ao[i % AHEAD], ot, i + AHEAD);
            else across(ao[i % AHEAD], qt, i + AHEAD - 2 * DT);
            if (i % 2 == 0 && i < 6) delta_of(i / 2 + 1);
#pragma unroll
            for (int e = 4 * i; e < 4 * i + 4; ++e) gradient(e);
            __builtin_amdgcn_sched_barrier(0);
        }
        // dK += Q^T dS beside the next step's first reads
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {
            const int slot = (i + 2 * DT) % AHEAD;
#pragma unroll
            for (int u = 0; u < 2; ++u) dk[u][i % DT] = T::mma(join<T>(ao[slot][0], ao[slot][1]), ds[u][i / DT], dk[u][i % DT]);
            if (i + AHEAD < 2 * DT) {
                across(ao[slot], qt, i + AHEAD);
            } else {                                    // this step's last reads are under way: the next one's first, and loads to where this one's rows were
                const int next = i + AHEAD - 2 * DT;
                if (next == 0) {
                    arrived<LOADS * (STAGES - 2)>();
                    load(s + STAGES, stage);
                }
                operand[next] = along(tiles[(stage.value + 1) % STAGES][0], next);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    static_assert(STAGES == 4);
    if (count) {
        load(0, std::integral_constant<int, 0>());
        load(1, std::integral_constant<int, 1>());
        load(2, std::integral_constant<int, 2>());
        arrived<LOADS * (STAGES - 2)>();
        load(3, std::integral_constant<int, 3>());
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) operand[i] = along(tiles[0][0], i);
    }
#pragma unroll 1
    for (uint32_t s = 0; s < count; s += 4) {
        step(s, std::integral_constant<int, 0>());
        if (s + 1 < count) step(s + 1, std::integral_constant<int, 1>());
        if (s + 2 < count) step(s + 2, std::integral_constant<int, 2>());
        if (s + 3 < count) step(s + 3, std::integral_constant<int, 3>());
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // nothing writes to shared memory any more when the block ends
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t key = key0 + 32 * u + n;
        const bool valid = key < tile.n;
        const int64_t at = (int64_t)tile.k0 + (valid ? key : 0);
        if (tile.pieces == 1) {
            store_row_16<T, DP>(a.dk + at * a.dks.token + tile.kvh * a.dks.head, valid, dk[u], a.scale, a.head_dim);
            store_row_16<T, DP>(a.dv + at * a.dvs.token + tile.kvh * a.dvs.head, valid, dv[u], 1.0f, a.head_dim);
        } else if (valid) {
            float *part = a.part_o + (tile.part(p, tile.piece) + 64 * wave + 32 * u + n) * 2 * DP;
            store_part<DP>(part, dk[u], a.scale);
            store_part<DP>(part + DP, dv[u], 1.0f);
        }
    }
}

// Sums of the pieces of tiles that were cut, in ascending order, rounded once: dQ of 32 rows a block, or, with KEYS, dK and dV of 32 keys.  Reads and writes
// alone: 57 MB of 8192 documents' keys in 13 us.
template <class T, int DP, int W, int STEP, bool KEYS>
__global__ __launch_bounds__(8 * DP) void k_prompt_sum(const PromptArgs p)
{
    constexpr int C4 = DP / 4 * (KEYS ? 2 : 1);
    const AttnArgs &a = p.a;
    Tile<32 * W, STEP, KEYS> tile(p, blockIdx.x / W, std::true_type());
    if (!tile.there) return;
    tile.settle();
    const uint32_t lines = KEYS ? tile.n : tile.m * a.group;
#pragma unroll
    for (uint32_t i = threadIdx.x; i < 32 * C4; i += 8 * DP) {
        const uint32_t within_tile = blockIdx.x % W * 32 + i / C4, own = tile.index * 32 * W + within_tile, c = i % C4, d = 4 * c % DP;
        if (own >= lines) return;
        if (d >= a.head_dim) continue;
        const int64_t line = tile.part(p, 0) + within_tile;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
        for (uint32_t s = 0; s < tile.pieces; ++s) x += *reinterpret_cast<const f32x4 *>(a.part_o + ((line + s * 32 * W) * C4 + c) * 4);
        uint16_t *to;
        if (!KEYS) to = a.dq + tile.q0 * a.dqs.token + row_at(a, a.dqs, 0, tile.kvh, own);
        else if (4 * c < DP) to = a.dk + (int64_t)(tile.k0 + own) * a.dks.token + tile.kvh * a.dks.head;
        else to = a.dv + (int64_t)(tile.k0 + own) * a.dvs.token + tile.kvh * a.dvs.head;
        *reinterpret_cast<typename T::V4 *>(to + d) = __builtin_convertvector(x, typename T::V4);
    }
}

}  // namespace mmee
