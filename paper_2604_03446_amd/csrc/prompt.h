// Attention of packed prompts: sequences of different lengths one behind the other, each row over its own sequence's keys, all of them or those
// up to its own.  Formulas, the folding of query heads into rows, the transposed scores and what is rounded are those of attention.h.
//
// A sequence's rows (for dK and dV its keys) are cut into tiles of a block each.  Blocks find theirs from the starts alone, and the host, which
// does not know the lengths, launches as many as any lengths can need, rows / TILE + seqs a head; those without a tile end at once.
//   Up to 64 sequences (a lane holds one): tiles in the order of their work, the longest first, whatever sequence they are of, so that the short
//   ones fill up the end; where there are few tiles, or some far longer than a unit's share, they are cut into pieces of equal length that are
//   joined afterwards (`pieces_of`).
//   More sequences: tile t of sequence b has slot (first row of b) / TILE + b + t, which differ whatever the lengths.
#pragma once

#include "attention.h"
#include "sequences.h"

namespace mmee {

struct PromptArgs {
    AttnArgs a;                 // batch 1, q_len: all tokens, rows: of all tokens, kv_len: all keys, splits: pieces of a tile at most
    const int32_t *q_starts, *kv_starts;
    uint32_t seqs, slots;
    uint32_t room_shift, least; // blocks that run at once (a power of two), steps of a piece at least
    bool causal;
    bool dies;                  // heads are dealt out to the dies, whose L2 then holds their keys
};

// A block's tile: rows (or, with KEYS, keys) index * TILE .. of a sequence of m tokens from q0 on over n keys from k0 on, and the steps step0 .. of
// STEP keys (or rows) that are the block's piece of it.
template <uint32_t TILE, uint32_t STEP, bool KEYS>
struct Tile {
    uint32_t index = 0, q0 = 0, m = 0, k0 = 0, n = 0, kvh, piece, pieces = 1, step0 = 0, count = 0;
    bool there = false;

    // at: place among heads, tiles and pieces.
    __device__ __forceinline__ Tile(const PromptArgs &p, uint32_t at)
    {
        piece = at % p.a.splits;
        at /= p.a.splits;
        const uint32_t order = at % p.slots;
        kvh = at / p.slots;
        uint32_t longest = p.least;                     // of a piece, in steps
        if (p.seqs <= 64) there = by_work(p, order, longest);
        else there = by_slot(p, p.slots - 1 - order);
        if (!there) return;
        const uint32_t steps = steps_of(p, m, n, index);
        if (p.a.splits > 1) {
            pieces = (steps + longest - 1) / longest;
            pieces = pieces < 1 ? 1 : pieces < p.a.splits ? pieces : p.a.splits;
        }
        const uint32_t per = pieces > 1 ? (steps + pieces - 1) / pieces : steps;
        step0 = piece * per < steps ? piece * per : steps;
        count = step0 + per < steps ? per : steps - step0;
        there = piece < pieces;
    }

    // Of a tile that is there: the same in all lanes, so that loops on its numbers are scalar, and so are the buffers that it is loaded from.  (Said once it is
    // known to be there; in the constructor, where lanes held numbers of their own, the compiler still made loops over the lanes of every load.)
    __device__ __forceinline__ void settle()
    {
        for (uint32_t *x : {&index, &q0, &m, &k0, &n, &kvh, &piece, &pieces, &step0, &count}) *x = __builtin_amdgcn_readfirstlane(*x);
    }

    static __device__ __forceinline__ uint32_t tiles_of(const PromptArgs &p, uint32_t m, uint32_t n) { return ((KEYS ? n : m * p.a.group) + TILE - 1) / TILE; }

    // Keys 0 .. that a token sees.
    static __device__ __forceinline__ uint32_t limit(const PromptArgs &p, uint32_t m, uint32_t n, uint32_t token)
    {
        return p.causal ? (uint32_t)within((int64_t)token + 1 + n - m, 0, n) : n;
    }

    // The first row that sees a key, which may lie before the first or behind the last one.
    static __device__ __forceinline__ int first_row(const PromptArgs &p, uint32_t m, uint32_t n, uint32_t key)
    {
        return p.causal ? (int)within(((int64_t)key + m - n) * p.a.group, -(1 << 29), (int64_t)m * p.a.group) : 0;
    }

    static __device__ __forceinline__ uint32_t steps_of(const PromptArgs &p, uint32_t m, uint32_t n, uint32_t index)
    {
        const uint32_t rows = m * p.a.group;
        if (KEYS) {
            const int begin = first_row(p, m, n, index * TILE);
            return (rows - (begin < 0 ? 0 : begin) + STEP - 1) / STEP;
        }
        const uint32_t behind = (index + 1) * TILE < rows ? (index + 1) * TILE : rows;
        return (limit(p, m, n, token_of(p.a, behind - 1)) + STEP - 1) / STEP;
    }

    __device__ __forceinline__ void take(const PromptArgs &p, uint32_t seq)
    {
        q0 = (uint32_t)within(p.q_starts[seq], 0, p.a.q_len);
        m = (uint32_t)within(p.q_starts[seq + 1], q0, p.a.q_len) - q0;
        k0 = (uint32_t)within(p.kv_starts[seq], 0, p.a.kv_len);
        n = (uint32_t)within(p.kv_starts[seq + 1], k0, p.a.kv_len) - k0;
    }

    __device__ __forceinline__ bool by_slot(const PromptArgs &p, uint32_t slot)
    {
        const int32_t *starts = KEYS ? p.kv_starts : p.q_starts;
        const uint32_t tokens = KEYS ? p.a.kv_len : p.a.q_len, each = KEYS ? 1 : p.a.group;
        const auto slot_of = [&](uint32_t i) { return (int64_t)((uint32_t)within(starts[i], 0, tokens) * each / TILE + i); };
        const int seq = __builtin_amdgcn_readfirstlane(last_at_most(p.seqs, slot, slot_of));
        if (seq < 0) return false;
        take(p, seq);
        index = slot - (uint32_t)slot_of(seq);
        return index < tiles_of(p, m, n);
    }

    // Tiles have levels, about their length in tiles: with a causal mask those of a sequence are neighbours, else they are the same.
    __device__ __forceinline__ bool by_work(const PromptArgs &p, uint32_t order, uint32_t &longest)
    {
        const uint32_t lane = threadIdx.x & 63;
        uint32_t tiles = 0, base = 0;
        if (lane < p.seqs) {
            take(p, lane);
            tiles = tiles_of(p, m, n);
            if (KEYS) base = p.causal ? 0 : m * p.a.group / STEP;
            else base = p.causal ? (n > m ? (n - m) * p.a.group / TILE : 0) : n / STEP;
        }
        if (order >= sum_of_lanes(tiles)) return false;
        // tiles of a sequence at this level or above
        const auto above = [&](uint32_t level) {
            if (!p.causal) return base >= level ? tiles : 0;
            return level <= base ? tiles : level < base + tiles ? base + tiles - level : 0;
        };
        uint32_t low = 0, high = p.seqs == 1 && p.causal ? base + tiles : most_of_lanes(p.causal ? base + tiles : base + 1);
        high = __builtin_amdgcn_readfirstlane(high);
        while (high - low > 1) {
            const uint32_t mid = (low + high) / 2;
            if (sum_of_lanes(above(mid)) > order) low = mid;
            else high = mid;
        }
        const uint32_t here = above(low) - above(low + 1), rank = order - sum_of_lanes(above(low + 1)), below = sums_below(here) - here;
        const uint64_t owner = __ballot(rank >= below && rank < below + here);
        const uint32_t seq = (uint32_t)__builtin_ctzll(owner);
        index = p.causal ? (KEYS ? tiles - 1 - (low - base) : low - base) : rank - below;
        if (p.a.splits > 1) longest = pieces_of(p, tiles);
        index = __builtin_amdgcn_readlane(index, seq);
        q0 = __builtin_amdgcn_readlane(q0, seq);
        m = __builtin_amdgcn_readlane(m, seq);
        k0 = __builtin_amdgcn_readlane(k0, seq);
        n = __builtin_amdgcn_readlane(n, seq);
        return true;
    }

    // The length that pieces may have: what each of the blocks that run at once gets of all steps.  Where there are fewer tiles than such blocks, the least
    // up to three times that with which all pieces run at once.  (The kernels that join the pieces come to the same ones: whole numbers, and products of
    // floats that nothing is added to.)
    __device__ __forceinline__ uint32_t pieces_of(const PromptArgs &p, uint32_t tiles) const
    {
        const uint32_t a = tiles ? steps_of(p, m, n, 0) : 0, b = tiles ? steps_of(p, m, n, tiles - 1) : 0;
        const uint32_t most = a > b ? a : b, least = a > b ? b : a;
        const uint32_t own = (uint32_t)((uint64_t)tiles * (a + b) >> 4);                // in 8 steps, on average over the tiles: below 2^31 in all
        const uint64_t share = (uint64_t)sum_of_lanes(own) * p.a.kv_heads * 8 >> p.room_shift, blocks = (uint64_t)sum_of_lanes(tiles) * p.a.kv_heads;
        const uint32_t low = share > p.least ? (uint32_t)share : p.least;
        if (blocks >> p.room_shift) return low;
        uint32_t no = low - 1, yes = 3 * low;
        while (yes - no > 1 + low / 16) {
            const uint32_t mid = (no + yes) / 2;
            const float inverse = 1.0f / (float)mid;
            const uint32_t wanted = most - least < mid ? tiles * ((most + mid - 1) / mid) : (uint32_t)((float)own * (8.0f * inverse)) + tiles / 2 + 1;
            if (((uint64_t)sum_of_lanes(tiles ? wanted : 0) * p.a.kv_heads - 1) >> p.room_shift == 0) yes = mid;
            else no = mid;
        }
        return yes;
    }

    // Keys of the sequence as the tiles' loads want them.
    __device__ __forceinline__ Keys<MODE_PLAIN> keys(const PromptArgs &p) const
    {
        Keys<MODE_PLAIN> k(p.a, 0, kvh);
        k.end = n;
        return k;
    }
};

__device__ __forceinline__ uint32_t block_place(const PromptArgs &p) { return p.dies ? by_die(blockIdx.x, gridDim.x) : blockIdx.x; }

// Scores of keys first + {8 (r / 4) + 4 h + r % 4} that a row with so many keys left does not see become -inf.
__device__ __forceinline__ void mask_behind(f32x16 &x, int left)
{
    const int own = left - 4 * (int)((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 8 * (r / 4) + r % 4 < own ? x[r] : -INFINITY;
}

// Forward: as k_attn_forward with W waves of 32 rows each on a tile of 64 keys, which ends where the block's last row does; only tiles that some row
// does not see whole are masked.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, 2) void k_prompt_forward(const PromptArgs p)
{
    constexpr int TN = 64, MT = 2, CH = DP / 8, GT = 64 * W;
    __shared__ u32x4 memory[4 * TN * CH];
    const AttnArgs &a = p.a;
    Tile<32 * W, TN, false> tile(p, block_place(p));
    if (!tile.there) return;
    tile.settle();
    const int thread = threadIdx.x, lane = thread & 63, n = lane & 31, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const uint32_t rows = tile.m * a.group, row0 = tile.index * 32 * W, row = row0 + 32 * wave + n, step0 = tile.step0, count = tile.count;
    const bool live = row < rows;
    const uint32_t limit = tile.limit(p, tile.m, tile.n, token_of(a, live ? row : rows - 1)), all_see = tile.limit(p, tile.m, tile.n, token_of(a, row0));

    const Keys<MODE_PLAIN> keys = tile.keys(p);
    const uint16_t *const k_at = a.k + tile.k0 * a.ks.token, *const v_at = a.v + tile.k0 * a.vs.token;
    typename T::V8 q[DP / 16];
    row_operands<T, DP>(q, a.q + tile.q0 * a.qs.token + row_at(a, a.qs, 0, tile.kvh, live ? row : 0), live, a.head_dim);

    f32x16 sums[1][DP / 32] = {};
    f32x16(&o)[DP / 32] = sums[0];
    float top = -INFINITY, total = 0.0f;                // mark near the maximum (scaled, in powers of two); this lane's share of the sum
    Stage<DP, TN, GT, MODE_PLAIN> sk, sv;
    auto k_tile = [&](uint32_t s) { return memory + (s & 1) * TN * CH; };
    auto v_tile = [&](uint32_t s) { return memory + (2 + (s & 1)) * TN * CH; };
    auto first_of = [&](uint32_t s) { return (step0 + s) * TN; };
    constexpr float HIGHER = NARROW<T> ? 7.0f : 0.0f;   // powers of two, of probabilities: see k_attn_forward
    f32x16 x[MT], ahead[MT];
    float most = -INFINITY;                             // maximum of the scores that are next, scaled

    auto load_keys = [&](uint32_t s) { sk.load(keys, k_at, a.ks, thread, first_of(s), 0); };
    auto load_values = [&](uint32_t s) { sv.load(keys, v_at, a.vs, thread, first_of(s), 0); };
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
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += now[mt][r];
            total += sum;
            to[mt][0][0] = rounded<T>(now[mt], 0);
            to[mt][1][0] = rounded<T>(now[mt], 1);
        }
    };
    auto values = [&](uint32_t s, const typename T::V8 (&of)[MT][2][1]) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int part = 0; part < 2; ++part) columns_times<T, DP, 1>(sums, v_tile(s), 32 * mt + 16 * part, of[mt][part]);
    };

    if (count) {
        // Tile s + 1's scores beside tile s's exponentials, its maximum beside tile s's product with V: K runs a tile ahead of V.
        load_keys(0);
        load_values(0);
        sk.store(k_tile(0), thread);
        sv.store(v_tile(0), thread);
        __syncthreads();
        load_keys(1);
        load_values(1);
        scores(x, 0);
        mask(x, 0);
        most = maximum(x);
        raise();
        sk.store(k_tile(1), thread);
        __syncthreads();
        load_keys(2);

        // Tile s from its scores `now`; unless it is the last, the next one's scores into `next`.
        auto step = [&](uint32_t s, f32x16 (&now)[MT], f32x16 (&next)[MT], auto more, auto masked) {
            typename T::V8 pr[MT][2][1];
            constexpr int PRODUCTS = MT * DP / 16;
            if (more) scores(next, s + 1);
            exponentials(now, pr);
            if (more) {
                // in one block of straight-line code: a product after every operand read and a share of the exponentials' work
                asm volatile("" ::"v"(total));
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int part = 0; part < 2; ++part) asm volatile("" ::"v"(pr[mt][part][0]));
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
                for (int i = 0; i < PRODUCTS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, (MT * 56 + PRODUCTS - 1) / PRODUCTS, 0);
                }
                if (masked) mask(next, s + 1);
            }
            values(s, pr);
            if (!more) return;
            most = maximum(next);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
#pragma unroll
            for (int i = 0; i < PRODUCTS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 1);
            }
            raise();
            sk.store(k_tile(s), thread);
            sv.store(v_tile(s + 1), thread);
            __syncthreads();
            load_keys(s + 3);
            load_values(s + 2);
        };
        uint32_t s = 0;
        for (; s + 3 < count && first_of(s + 3) <= all_see; s += 2) {       // tiles s + 1 and s + 2 are seen whole by every row
            step(s, x, ahead, std::true_type(), std::false_type());
            step(s + 1, ahead, x, std::true_type(), std::false_type());
        }
#pragma unroll 1
        for (; s + 1 < count; ++s) {
            step(s, x, ahead, std::true_type(), std::true_type());
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) x[mt] = ahead[mt];
        }
        step(s, x, ahead, std::false_type(), std::false_type());
    }
    total = sum_of_halves(total);
    if (!live) return;
    const float times = total != 0.0f ? 1.0f / total : 0.0f, sum2 = total != 0.0f ? top + __log2f(total) : -INFINITY;
    if (tile.pieces == 1) {
        store_row<T, DP>(a.o + tile.q0 * a.os.token + row_at(a, a.os, 0, tile.kvh, row), o, times, a.head_dim);
        if (a.lse && h == 0) a.lse[lse_at(a, 0, tile.kvh, row) + tile.q0] = sum2 * LN2;
    } else {
        const int64_t line = ((int64_t)tile.piece * a.kv_heads + tile.kvh) * a.rows + tile.q0 * a.group + row;
        store_part<DP>(a.part_o + line * DP, o, times);
        if (h == 0) a.part_lse[line] = sum2;
    }
}

// Joins the pieces of the tiles of 32 W rows that were cut, in ascending order, as k_attn_join does: 32 rows a block.
template <class T, int DP, int W>
__global__ __launch_bounds__(256) void k_prompt_join(const PromptArgs p)
{
    constexpr int C4 = DP / 4;
    const AttnArgs &a = p.a;
    Tile<32 * W, 64, false> tile(p, blockIdx.x / W * a.splits);
    if (!tile.there || tile.pieces == 1) return;
    tile.settle();
    const int64_t next = (int64_t)a.kv_heads * a.rows;
    for (uint32_t i = threadIdx.x; i < 32 * C4; i += 256) {
        const uint32_t row = tile.index * 32 * W + blockIdx.x % W * 32 + i / C4, c = i % C4;
        if (row >= tile.m * a.group) return;
        const int64_t line = (int64_t)tile.kvh * a.rows + tile.q0 * a.group + row;
        float high = -INFINITY, sum = 0.0f;
        for (uint32_t s = 0; s < tile.pieces; ++s) high = __builtin_elementwise_maximum(high, a.part_lse[s * next + line]);
        const float off = high == -INFINITY ? 0.0f : high;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
        for (uint32_t s = 0; s < tile.pieces; ++s) {
            const float w = __builtin_amdgcn_exp2f(a.part_lse[s * next + line] - off);
            sum += w;
            x += *reinterpret_cast<const f32x4 *>(a.part_o + (s * next + line) * DP + 4 * c) * w;
        }
        x *= sum != 0.0f ? 1.0f / sum : 0.0f;
        if (4 * c < a.head_dim) *reinterpret_cast<typename T::V4 *>(a.o + tile.q0 * a.os.token + row_at(a, a.os, 0, tile.kvh, row) + 4 * c) = __builtin_convertvector(x, typename T::V4);
        if (a.lse && c == 0) a.lse[lse_at(a, 0, tile.kvh, row) + tile.q0] = sum != 0.0f ? (high + __log2f(sum)) * LN2 : -INFINITY;
    }
}

// dQ, and D on the way, as k_attn_dq.
template <class T, int DP, int W>
__global__ __launch_bounds__(64 * W, 2) void k_prompt_dq(const PromptArgs p)
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
    const uint32_t limit = tile.limit(p, tile.m, tile.n, token_of(a, live ? row : rows - 1));

    const Keys<MODE_PLAIN> keys = tile.keys(p);
    const uint16_t *const k_at = a.k + tile.k0 * a.ks.token, *const v_at = a.v + tile.k0 * a.vs.token;
    const int64_t line = (int64_t)tile.kvh * a.rows + tile.q0 * a.group + row;
    typename T::V8 q[DP / 16], d_o[DP / 16];
    row_operands<T, DP>(q, a.q + tile.q0 * a.qs.token + row_at(a, a.qs, 0, tile.kvh, live ? row : 0), live, a.head_dim);
    row_operands<T, DP>(d_o, a.d_o + tile.q0 * a.dos.token + row_at(a, a.dos, 0, tile.kvh, live ? row : 0), live, a.head_dim);
    float lse2 = INFINITY, delta = 0.0f;                // rows that see nothing: probabilities 0
    if (live) {
        const float l = a.lse_in[lse_at(a, 0, tile.kvh, row) + tile.q0];
        lse2 = l == -INFINITY ? INFINITY : l * LOG2E - (NARROW<T> ? UP + HIGHEST : 0.0f);
    }
    {
        typename T::V8 o[DP / 16];
        row_operands<T, DP>(o, a.o_in + tile.q0 * a.os.token + row_at(a, a.os, 0, tile.kvh, live ? row : 0), live, a.head_dim);
#pragma unroll
        for (int t = 0; t < DP / 16; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta += (float)o[t][j] * (float)d_o[t][j];
        delta = sum_of_halves(delta);
        if (live && h == 0 && tile.piece == 0) a.delta[line] = delta;
    }

    f32x16 dq[1][DP / 32] = {};
    float lowered = 0.0f;                               // of dS's power of two, which lse2 holds
    Stage<DP, TN, 64 * W, MODE_PLAIN> sk, sv;
    auto first_of = [&](uint32_t s) { return (step0 + s) * TN; };
    if (count) {
        sk.load(keys, k_at, a.ks, thread, first_of(0), 0);
        sv.load(keys, v_at, a.vs, thread, first_of(0), 0);
    }
    for (uint32_t s = 0; s < count; ++s) {
        u32x4 *kt = tiles[s & 1][0], *vt = tiles[s & 1][1];
        sk.store(kt, thread);
        sv.store(vt, thread);
        __syncthreads();
        if (s + 1 < count) {
            sk.load(keys, k_at, a.ks, thread, first_of(s + 1), 0);
            sv.load(keys, v_at, a.vs, thread, first_of(s + 1), 0);
        }
        const int left = (int)limit - (int)first_of(s);
        const bool whole = __all(left >= TN);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            f32x16 x = keys_by_rows<T, DP>(kt, 32 * mt, q);
            const f32x16 dp = keys_by_rows<T, DP>(vt, 32 * mt, d_o);
            if (!whole) mask_behind(x, left - 32 * mt);
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale_log2, -lse2)) * (dp[r] - delta);
            if (NARROW<T>) {
                const float by = keep_in_range(x, dq[0]);
                lowered += by;
                lse2 -= by;
            }
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const typename T::V8 ds[1] = {rounded<T>(x, part)};
                columns_times<T, DP, 1>(dq, kt, 32 * mt + 16 * part, ds);
            }
        }
    }
    if (!live) return;
    if (lse2 == INFINITY) {                             // (a row that sees nothing, whatever its query and gradient hold)
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt) dq[0][dt] = f32x16{};
    }
    const float times = NARROW<T> ? a.scale * __builtin_amdgcn_exp2f(-(UP + HIGHEST + lowered)) : a.scale;
    if (tile.pieces == 1) store_row<T, DP>(a.dq + tile.q0 * a.dqs.token + row_at(a, a.dqs, 0, tile.kvh, row), dq[0], times, a.head_dim);
    else store_part<DP>(a.part_o + ((int64_t)tile.piece * a.kv_heads * a.rows + line) * DP, dq[0], times);
}

// dK and dV of 32 W keys, 32 a wave, over the rows that see them, as k_attn_dkv.
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
    const int own = tile.first_row(p, tile.m, tile.n, key), all_see = tile.first_row(p, tile.m, tile.n, key0 + 32 * W - 1);
    const int first_seen = tile.first_row(p, tile.m, tile.n, key0);
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
        }
    }
    if (!valid) return;
    const float times = NARROW<T> ? a.scale * 0x1p-15f / by : a.scale, times_v = NARROW<T> ? 0x1p-15f : 1.0f;
    if (tile.pieces == 1) {
        store_row<T, DP>(a.dk + key_at * a.dks.token + tile.kvh * a.dks.head, dk[0], times, a.head_dim);
        store_row<T, DP>(a.dv + key_at * a.dvs.token + tile.kvh * a.dvs.head, dv[0], times_v, a.head_dim);
    } else {
        float *part = a.part_o + ((((int64_t)tile.piece * a.kv_heads + tile.kvh) * a.kv_len + key_at) * 2) * DP;
        store_part<DP>(part, dk[0], times);
        store_part<DP>(part + DP, dv[0], times_v);
    }
}

// Sums of the pieces of tiles that were cut, in ascending order, rounded once, as k_attn_sum: dQ of 32 rows a block, or, with KEYS, dK and dV of 32 keys.
template <class T, int DP, int W, int STEP, bool KEYS>
__global__ __launch_bounds__(256) void k_prompt_sum(const PromptArgs p)
{
    constexpr int C4 = DP / 4 * (KEYS ? 2 : 1);
    const AttnArgs &a = p.a;
    Tile<32 * W, STEP, KEYS> tile(p, blockIdx.x / W * a.splits);
    if (!tile.there || tile.pieces == 1) return;
    tile.settle();
    const uint32_t lines = KEYS ? tile.n : tile.m * a.group;
    const int64_t next = (int64_t)a.kv_heads * (KEYS ? a.kv_len : a.rows);
    for (uint32_t i = threadIdx.x; i < 32 * C4; i += 256) {
        const uint32_t own = tile.index * 32 * W + blockIdx.x % W * 32 + i / C4, c = i % C4, d = 4 * c % DP;
        if (own >= lines) return;
        if (d >= a.head_dim) continue;
        const int64_t line = KEYS ? (int64_t)tile.kvh * a.kv_len + tile.k0 + own : (int64_t)tile.kvh * a.rows + tile.q0 * a.group + own;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
        for (uint32_t s = 0; s < tile.pieces; ++s) x += *reinterpret_cast<const f32x4 *>(a.part_o + ((s * next + line) * C4 + c) * 4);
        uint16_t *to;
        if (!KEYS) to = a.dq + tile.q0 * a.dqs.token + row_at(a, a.dqs, 0, tile.kvh, own);
        else if (4 * c < DP) to = a.dk + (int64_t)(tile.k0 + own) * a.dks.token + tile.kvh * a.dks.head;
        else to = a.dv + (int64_t)(tile.k0 + own) * a.dvs.token + tile.kvh * a.dvs.head;
        *reinterpret_cast<typename T::V4 *>(to + d) = __builtin_convertvector(x, typename T::V4);
    }
}

}  // namespace mmee
