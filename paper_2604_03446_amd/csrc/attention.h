// Attention of rows of queries over keys of another length: forward, over plain tensors or over a paged cache with a tree of
// drafted tokens, and backward.
//
//   S = scale Q K^T, masked entries -inf;  P = softmax(S);  O = P V;  lse = log sum exp S
//   D = rowsum(dO * O);  dV = P^T dO;  dS = P (dO V^T - D);  dQ = scale dS K;  dK = scale dS^T Q
//
// The query heads that share a key/value head are rows of one problem: row r = token * group + head in group, so one tile of keys
// serves them all, and dK, dV sum over them without another pass.  Scores are formed transposed (keys along the matrix
// instruction's m, rows along n): a lane holds one row's scores, the softmax needs one exchange between two lanes, and the
// probabilities are the next product's operand as they stand.  Products take 16-bit operands and accumulate in 32 bits; maximum, sum,
// accumulators, lse, D and partial results are 32 bits; probabilities and dS are rounded to the operands' type, as the matrix
// instructions need them.
#pragma once

#include "launch.h"
#include "mfma.h"

namespace mmee {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Strides {                // in elements
    int64_t batch, token, head;
};

struct AttnArgs {
    const uint16_t *q, *k, *v;
    Strides qs, ks, vs, os;     // of pages: batch is the page's stride
    uint16_t *o;
    float *lse;                 // [batch][heads][q_len] or null
    uint32_t batch, heads, kv_heads, group, q_len, rows, kv_len, head_dim;
    uint64_t group_inverse;     // ceil(2^group_shift / group)
    uint32_t group_shift;
    float scale, scale_log2;
    const int32_t *kv_lens;
    const uint8_t *key_mask;
    int64_t mask_stride;
    // paged cache and tree
    const int32_t *page_table, *cache_lens, *node_counts;
    const uint64_t *ancestors;
    int64_t table_stride;
    uint32_t page_shift, n_pages, words;
    // keys in pieces
    uint32_t row_tiles, splits;         // splits: pieces of every sequence
    uint32_t slots, step_keys, least;   // forward: room for pieces of all sequences, keys of a step, steps of a piece at least
    bool balanced;                      // forward: pieces by the sequences' lengths, not `splits` of each
    uint32_t *cut;              // forward, balanced: every sequence's pieces and first slot, for the join
    float *part_o, *part_lse;   // forward [slot][kv_head][row][DP], [..][row], lse in powers of two; backward [split][batch][kv_head][row or key]..
    // backward
    const uint16_t *d_o, *o_in;
    const float *lse_in;
    Strides dos, dqs, dks, dvs;
    uint16_t *dq, *dk, *dv;
    float *delta;               // [batch][kv_head][row]
};

enum { MODE_PLAIN = 0, MODE_MASK = 1, MODE_TREE = 2 };

__device__ __forceinline__ uint32_t token_of(const AttnArgs &a, uint32_t row) { return (uint32_t)((row * a.group_inverse) >> a.group_shift); }

// Place of a row in a tensor of query heads.
__device__ __forceinline__ int64_t row_at(const AttnArgs &a, const Strides &s, uint32_t b, uint32_t kvh, uint32_t row)
{
    const uint32_t token = token_of(a, row), head = kvh * a.group + (row - token * a.group);
    return b * s.batch + token * s.token + head * s.head;
}

__device__ __forceinline__ int64_t lse_at(const AttnArgs &a, uint32_t b, uint32_t kvh, uint32_t row)
{
    const uint32_t token = token_of(a, row), head = kvh * a.group + (row - token * a.group);
    return ((int64_t)b * a.heads + head) * a.q_len + token;
}

__device__ __forceinline__ u32x4 zeros() { return u32x4{0, 0, 0, 0}; }

// Eight values of a row, as a B operand along the head's dimension: chunk 2 t + h of lane 32 h + i.
template <class T, int DP>
__device__ __forceinline__ void row_operands(typename T::V8 (&out)[DP / 16], const uint16_t *row, bool valid, uint32_t head_dim)
{
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) {
        const int at = 16 * t + 8 * h;
        out[t] = as_operand<T>(valid && at < (int)head_dim ? *reinterpret_cast<const u32x4 *>(row + at) : zeros());
    }
}

// Where the keys of a block's piece lie, and which of them count.
template <int MODE>
struct Keys {
    const AttnArgs &a;
    uint32_t b, kvh;
    uint32_t end;               // keys 0 .. end-1 exist
    uint32_t held, nodes;       // tree: keys in the cache before the tree, nodes
    uint32_t first_token = 0, last_token = 0;           // tree: nodes whose rows the block has, from the first one to behind the last one

    // Keys of sequence b; of a tree also those before it and the nodes.
    static __device__ __forceinline__ uint32_t length(const AttnArgs &a, uint32_t b, uint32_t &held, uint32_t &nodes)
    {
        if (MODE == MODE_TREE) {
            const int64_t room = (int64_t)a.kv_len;
            const int64_t len = a.cache_lens[b], n = a.node_counts ? a.node_counts[b] : (int32_t)a.q_len;
            held = (uint32_t)(len < 0 ? 0 : len > room ? room : len);
            nodes = (uint32_t)(n < 0 ? 0 : n > (int64_t)a.q_len ? (int64_t)a.q_len : n);
            if (!nodes || !a.n_pages) return 0;         // no row looks at anything
            return held + nodes > a.kv_len ? a.kv_len : held + nodes;
        }
        if (!a.kv_lens) return a.kv_len;
        const int32_t len = a.kv_lens[b];
        return len < 0 ? 0 : (uint32_t)len < a.kv_len ? (uint32_t)len : a.kv_len;
    }

    __device__ __forceinline__ Keys(const AttnArgs &args, uint32_t b_, uint32_t kvh_) : a(args), b(b_), kvh(kvh_), held(0), nodes(0)
    {
        end = length(a, b, held, nodes);
        end = __builtin_amdgcn_readfirstlane(end);      // the same in all lanes: loops and branches on it are scalar
        held = __builtin_amdgcn_readfirstlane(held);
        nodes = __builtin_amdgcn_readfirstlane(nodes);
    }

    // What decides whether key `at` counts: its page, or -1, and of a node who sees it; its mask byte.  Not asked where there are no keys.
    __device__ __forceinline__ int info(uint32_t at) const
    {
        if (MODE == MODE_PLAIN) return 0;
        const uint32_t key = at < end ? at : end - 1;   // (there is one at least)
        if (MODE == MODE_MASK) return a.key_mask[b * a.mask_stride + key] && at < end ? 0 : -1;
        const int32_t page = a.page_table[b * a.table_stride + (key >> a.page_shift)];
        bool counts = at < end;
        if (counts && key >= held) {
            // A node that no row sees does not count: its values may be anything, and a probability of 0 does not clear what is infinite or
            // NaN.  As a rule a node sees itself, so that its own row answers; for pruned ones the block's rows are asked, sixteen at a time.  (Seven
            // nodes over 500 keys: 0.7 us of 12.1; many nodes: none.  All rows' bits joined beforehand, or the stored tile looked through for
            // such values: 1.2 to 1.9.  44 of 64 nodes pruned: 4 % more; 924 of 1024 over
            // 700 keys, 8 heads: 151 us, which a count of nodes instead of empty rows spares, 66 if nothing were asked.)
            const uint32_t j = key - held;
            const uint64_t *column = a.ancestors + (int64_t)b * a.q_len * a.words + (j >> 6);
            counts = column[j * a.words] >> (j & 63) & 1;
#pragma unroll 1
            for (uint32_t i = first_token; i < last_token && !counts; i += 16) {
                uint64_t some = 0;
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) some |= column[(i + k < last_token ? i + k : i) * a.words];
                counts = some >> (j & 63) & 1;
            }
        }
        return (uint32_t)page < a.n_pages && counts ? page : -1;
    }
};

// How many pieces the forward pass cuts each of up to 64 sequences into: lane b has sequence b's number and its first slot.  Pieces have
// as nearly as possible the same number of steps, the least P for which all of them fit the slots: blocks of one round then end
// together whatever the lengths.  64 values of P between total / slots and three times that are tried at once.
template <int MODE>
__device__ __forceinline__ void balance(const AttnArgs &a, uint32_t &pieces, uint32_t &first_slot)
{
    const uint32_t lane = threadIdx.x & 63;
    uint32_t held, nodes;
    const uint32_t steps = lane < a.batch ? (Keys<MODE>::length(a, lane, held, nodes) + a.step_keys - 1) / a.step_keys : 0;
    uint32_t total = steps;
#pragma unroll
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    const uint32_t low = (total + a.slots - 1) / a.slots, least = low > a.least ? low : a.least;
    const uint32_t p = least + (uint32_t)(((uint64_t)least * lane + 31) / 32);
    uint32_t wanted = 0;
    for (uint32_t b = 0; b < a.batch; ++b) {
        const uint32_t of = __builtin_amdgcn_readlane(steps, b);
        wanted += of ? (of + p - 1) / p : 1;
    }
    const uint64_t fits = __ballot(wanted <= a.slots);
    const uint32_t size = fits ? __builtin_amdgcn_readlane(p, __builtin_ctzll(fits)) : 0;
    pieces = lane < a.batch ? (size && steps ? (steps + size - 1) / size : 1) : 0;
    uint32_t sum = pieces;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t below = __shfl_up(sum, d);
        sum += lane >= (uint32_t)d ? below : 0;
    }
    first_slot = sum - pieces;
}

// One thread's share of a tile of TN keys' K or V by GT threads: loads in flight in registers, then to shared memory.  Keys past the last one and
// columns past the head's are zeros, as are masked keys, which may hold anything, and those of pages that are not there: a probability or a
// row's operand of 0 does not clear what is infinite or NaN.  What does not exist is asked for beyond the buffer's end, so that nothing branches.
template <int DP, int TN, int GT, int MODE>
struct Stage {
    static constexpr int CH = DP / 8, LOADS = TN * CH / GT, ROWS = GT / CH;     // rows that one load of all threads covers
    static_assert(LOADS * GT == TN * CH && ROWS * CH == GT, "a tile is dealt out evenly");
    u32x4 r[LOADS];
    bool there[MODE == MODE_TREE ? LOADS : 1];
    uint64_t which;                     // MODE_MASK: the tile's keys that count, one bit each
    float bias;                         // MODE_MASK: 0 or -inf, for key first + (lane mod TN)

    // info: of key first + (lane mod TN), as Keys::info gives it.  There is a key at least.
    __device__ __forceinline__ void load(const Keys<MODE> &keys, const uint16_t *from, const Strides &s, int thread, uint32_t first, int info)
    {
        const AttnArgs &a = keys.a;
        const int row0 = thread / CH, c = thread % CH;
        const bool inside = 8 * c < (int)a.head_dim;
        if (MODE == MODE_TREE) {
            // a lane works out where its key lies; the threads that load the key ask it
            const uint32_t key = first + (threadIdx.x & 63) % TN, within = key & ((1u << a.page_shift) - 1);
            const int64_t place = info >= 0 ? info * s.batch + within * s.token : -1;
            const uint16_t *base = from + keys.kvh * s.head + (inside ? c * 8 : 0);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int row = row0 + i * ROWS, high = __shfl((int)(place >> 32), row);
                const uint32_t low = __shfl((uint32_t)place, row);
                there[MODE == MODE_TREE ? i : 0] = high >= 0 && inside;
                r[i] = *reinterpret_cast<const u32x4 *>(base + (high >= 0 ? (int64_t)high << 32 | low : 0));
            }
            return;
        }
        const uint32_t begin = first < keys.end ? first : keys.end, left = keys.end - begin;
        const auto base = buffer_at(from + keys.b * s.batch + keys.kvh * s.head + begin * s.token);
        const uint32_t step = 2 * (uint32_t)s.token, column = inside ? 16 * c : BEYOND;         // a tile spans less than 2^31 bytes
        if (MODE == MODE_MASK) {
            which = __ballot(info >= 0);
            bias = info >= 0 ? 0.0f : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t row = row0 + i * ROWS;
            r[i] = __builtin_amdgcn_raw_buffer_load_b128(base, row < left ? row * step + column : BEYOND, 0, 0);
        }
    }

    __device__ __forceinline__ void store(u32x4 *tile, int thread) const
    {
        const int c = thread % CH, row0 = thread / CH;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            bool counts = true;
            if (MODE == MODE_TREE) counts = there[MODE == MODE_TREE ? i : 0];
            if (MODE == MODE_MASK) counts = ROWS <= 32 ? (uint32_t)(which >> (i * ROWS % 64)) >> row0 & 1 : which >> row0 & 1;
            tile[chunk_at<CH>(row0 + i * ROWS, c)] = counts ? r[i] : zeros();
        }
    }
};

// S^T of 32 keys (rows `first` .. of a tile) and the wave's 32 rows, on top of s.
template <class T, int DP>
__device__ __forceinline__ f32x16 keys_by_rows(const u32x4 *tile, int first, const typename T::V8 (&rows)[DP / 16], f32x16 s = {})
{
    constexpr int CH = DP / 8;
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) s = T::mma(as_operand<T>(tile[first * CH + chunk_at<CH>(i, 2 * t + h)]), rows[t], s);
    return s;
}

// acc[u][dt] += (columns 32 dt .. of the tile's rows first .. first+15)^T times operands that hold these rows in the order of a
// 32x32 result: rows 4 h + {0..3}, 8 + 4 h + {0..3} in lane 32 h + i.
template <class T, int DP, int N>
__device__ __forceinline__ void columns_times(f32x16 (&acc)[N][DP / 32], const u32x4 *tile, int first, const typename T::V8 (&p)[N])
{
    constexpr int CH = DP / 8;
    const int lane = threadIdx.x & 63, i = lane & 15, g = (lane >> 4) & 1, h = lane >> 5;
    const char *base = reinterpret_cast<const char *>(tile + first * CH) + 8 * (i & 1);
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt) {
        const int c = 4 * dt + 2 * g + ((i >> 1) & 1), row = 4 * h + (i >> 2);
        const s16x4 lo = read_transposed(base + 16 * chunk_at<CH>(row, c)), hi = read_transposed(base + 16 * chunk_at<CH>(row + 8, c));
#pragma unroll
        for (int u = 0; u < N; ++u) acc[u][dt] = T::mma(join<T>(lo, hi), p[u], acc[u][dt]);
    }
}

template <class T>
__device__ __forceinline__ typename T::V8 rounded(const f32x16 &x, int part)
{
    f32x8 y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[8 * part + j];
    return __builtin_convertvector(y, typename T::V8);
}

// Stores a lane's column of a transposed result: values 32 dt + 8 u + 4 h + {0..3} of one row.
template <class T, int DP>
__device__ __forceinline__ void store_row(uint16_t *row, const f32x16 (&acc)[DP / 32], float times, uint32_t head_dim)
{
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int d = 32 * dt + 8 * u + 4 * h;
            const f32x4 x = {acc[dt][4 * u] * times, acc[dt][4 * u + 1] * times, acc[dt][4 * u + 2] * times, acc[dt][4 * u + 3] * times};
            if (d < (int)head_dim) *reinterpret_cast<typename T::V4 *>(row + d) = __builtin_convertvector(x, typename T::V4);
        }
}

template <int DP>
__device__ __forceinline__ void store_part(float *row, const f32x16 (&acc)[DP / 32], float times)
{
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const f32x4 x = {acc[dt][4 * u] * times, acc[dt][4 * u + 1] * times, acc[dt][4 * u + 2] * times, acc[dt][4 * u + 3] * times};
            *reinterpret_cast<f32x4 *>(row + 32 * dt + 8 * u + 4 * h) = x;
        }
}

// Scores of 32 keys whose bits say that the key does not count become -inf.  The same keys for all rows: the lanes' masks are formed in
// scalar registers.
__device__ __forceinline__ void mask_keys(f32x16 &x, uint32_t bits)
{
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r / 4) + r % 4;            // in the lower half of the lanes; 4 more in the upper one
        const uint32_t low = -(int)(bits >> key & 1), high = -(int)(bits >> (key + 4) & 1);
        x[r] = __builtin_amdgcn_inverse_ballot_w64((uint64_t)high << 32 | low) ? x[r] : -INFINITY;
    }
}

// What the products of 32 masked keys start from: 0, or -inf for keys that do not count (whose K is zeros).  It costs four reads and no
// vector instruction; selecting afterwards took 25 % longer at 64 values a head.
__device__ __forceinline__ f32x16 biases(const float *of)
{
    const int h = (threadIdx.x >> 5) & 1;
    f32x16 x;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 four = *reinterpret_cast<const f32x4 *>(of + 8 * g + 4 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * g + j] = four[j];
    }
    return x;
}

// Keys of a tile that exist and count, one bit each.
template <int MODE, int TN>
__device__ __forceinline__ uint64_t counted(const Keys<MODE> &keys, uint32_t first, int info)
{
    constexpr uint64_t WHOLE = ~0ull >> (64 - TN);
    if (MODE != MODE_PLAIN) return __ballot(info >= 0) & WHOLE;
    const uint32_t left = keys.end > first ? keys.end - first : 0;
    return left >= TN ? WHOLE : (1ull << left) - 1;
}

// Those of them that a lane's row of a tree sees.
template <int TN>
__device__ __forceinline__ uint64_t seen(const Keys<MODE_TREE> &keys, uint32_t first, uint64_t bits, uint32_t token)
{
    const AttnArgs &a = keys.a;
    if (token >= keys.nodes) return 0;
    if (first + TN <= keys.held) return bits;
    const uint64_t *words = a.ancestors + ((int64_t)keys.b * a.q_len + token) * a.words;
    const int64_t j = (int64_t)first - keys.held;       // > -64
    if (j < 0) return bits & (words[0] << -j | ((1ull << -j) - 1));
    const uint32_t w = (uint32_t)(j >> 6), by = (uint32_t)(j & 63);
    if (w >= a.words) return 0;
    uint64_t own = words[w] >> by;
    if (by && w + 1 < a.words) own |= words[w + 1] << (64 - by);
    return bits & own;
}

// Forward.  WR waves share a tile of keys, 32 rows each; WK such groups take every WK-th tile of the block's piece and are joined
// at the end.  WR = 4 or 8 for many rows: a tile serves 128 or 256.  WK = 4 or 8 for 32 rows or fewer (single tokens): nothing is shared
// between waves and no barrier is met while keys stream in.
//
// Many rows are bound by the compute unit: of a step's 2.1 us the matrix instructions need 0.85, the reads of operands from shared memory
// 0.85 and the vector instructions 0.9, and they overlap in part.  2048 rows over 8192 keys, 32 heads of 128: 257 to 280 us, 1.0 PFLOP/s
// (a library product of 16-bit matrices reaches 1.39); 2 x 2048 over 4096, 32 heads over 8: 278 to 300 us, 0.95.  With a mask of a byte a key, 8 x
// 509 rows over 1500, 12 heads of 64: 47 to 50 us, 0.4 PFLOP/s: an exponential a score weighs twice as much as with 128 values a head.  Sixteen
// trees of up to 63 nodes over contexts of 2048 to 4096 in pages of 16, 32 heads over 8: 94 us, where every block streams keys that no other
// one reads: 2.4 TB/s and 0.56 PFLOP/s at once; 26 nodes over contexts up to 131072, 64 heads over 8: 309 to 375 us, 2.1 to 2.6 TB/s.
// With 128 values a head all 256 registers of a wave are in use: eight waves without a mask spill 3 or 4 more, four waves with a mask or a tree 10 to 14.
// Few rows are bound by HBM: 64 tokens over 1024 to 2048 keys, 32 heads over 8: 82 us, 4.9 TB/s; one token over 512 keys, 12 heads: 6 us,
// the latency of a launch, of the lengths, the keys and the join.
template <class T, int DP, int WR, int WK, int MODE>
__global__ __launch_bounds__(64 * WR * WK, 2) void k_attn_forward(const AttnArgs a)
{
    constexpr int TN = WR >= 4 ? 64 : 32, MT = TN / 32, CH = DP / 8, GT = 64 * WR, NB = WR >= 4 ? 2 : 1, TILES = 2 * NB * WK * TN * CH;
    static_assert(NB == 1 || WK == 1, "two buffers for one group");
    constexpr int JOIN = WK > 1 ? WK * 32 * WR * DP / 4 : 0;
    __shared__ u32x4 memory[TILES > JOIN ? TILES : JOIN];
    __shared__ float marks[2][WK][WK > 1 ? 32 * WR : 1];
    __shared__ __align__(16) float bias[WK][NB][MODE == MODE_MASK ? TN : 4];
    const int thread = threadIdx.x % GT, lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave % WR, wk = wave / WR;      // scalar: the tiles' places are

    uint32_t at = by_die(blockIdx.x, gridDim.x);
    const uint32_t rt = at % a.row_tiles;
    at /= a.row_tiles;
    const uint32_t kvh = at % a.kv_heads, slot = at / a.kv_heads;
    uint32_t b = slot / a.splits, split = slot % a.splits, pieces = a.splits;
    if (a.balanced) {
        uint32_t n, first;
        balance<MODE>(a, n, first);
        if (blockIdx.x == 0 && threadIdx.x < a.batch) {
            a.cut[2 * threadIdx.x] = n;
            a.cut[2 * threadIdx.x + 1] = first;
        }
        const uint64_t owner = __ballot(slot >= first && slot < first + n);
        if (!owner) return;                             // by the whole block
        b = __builtin_ctzll(owner);
        pieces = __builtin_amdgcn_readlane(n, b);
        split = slot - __builtin_amdgcn_readlane(first, b);
    }
    Keys<MODE> keys(a, b, kvh);
    // pieces of whole steps (TN keys for every group)
    constexpr uint32_t STEP = TN * WK;
    const uint32_t steps = (keys.end + STEP - 1) / STEP, per = (steps + pieces - 1) / pieces;
    const uint32_t step0 = split * per < steps ? split * per : steps, count = step0 + per < steps ? per : steps - step0;

    const uint32_t row = (rt * WR + wr) * 32 + n;
    const bool live = row < a.rows;
    const uint32_t token = token_of(a, live ? row : 0);
    if (MODE == MODE_TREE) {
        const uint32_t behind = (rt + 1) * WR * 32 < a.rows ? (rt + 1) * WR * 32 : a.rows, last = token_of(a, behind - 1) + 1;
        keys.first_token = token_of(a, rt * WR * 32);
        keys.last_token = last < keys.nodes ? last : keys.nodes;
    }
    typename T::V8 q[DP / 16];
    row_operands<T, DP>(q, a.q + (live ? row_at(a, a.qs, b, kvh, row) : 0), live, a.head_dim);

    f32x16 sums[1][DP / 32] = {};
    f32x16(&o)[DP / 32] = sums[0];
    float top = -INFINITY, total = 0.0f;                // mark near the maximum (scaled, in powers of two); this lane's share of the sum

    Stage<DP, TN, GT, MODE> sk, sv;
    u32x4 *const mine = memory + wk * 2 * NB * TN * CH;
    auto k_tile = [&](uint32_t s) { return mine + (NB == 2 ? s & 1 : 0) * TN * CH; };
    auto v_tile = [&](uint32_t s) { return mine + (NB + (NB == 2 ? s & 1 : 0)) * TN * CH; };
    auto first_of = [&](uint32_t s) { return ((step0 + s) * WK + wk) * TN; };
    auto info_of = [&](uint32_t s) { return keys.info(first_of(s) + lane % TN); };
    auto sync = [&] { if (WR > 1) __syncthreads(); else wave_sync(); };
    constexpr uint64_t WHOLE = ~0ull >> (64 - TN);
    constexpr float HIGHER = NARROW<T> ? 7.0f : 0.0f;   // powers of two, of probabilities
    f32x16 x[MT];
    float most = -INFINITY;                             // maximum of the scores that are next, scaled
    int info[3] = {};                                   // of the tile whose scores come next and the two behind it

    auto scores = [&](f32x16 (&to)[MT], uint32_t s) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            to[mt] = keys_by_rows<T, DP>(k_tile(s), 32 * mt, q, MODE == MODE_MASK ? biases(bias[wk][NB == 2 ? s & 1 : 0] + (MODE == MODE_MASK ? 32 * mt : 0)) : f32x16{});
    };
    auto mask = [&](f32x16 (&to)[MT], uint32_t s) {
        if (MODE == MODE_MASK) return;
        const uint64_t bits = counted<MODE, TN>(keys, first_of(s), info[0]);
        if constexpr (MODE != MODE_TREE) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) mask_keys(to[mt], (uint32_t)(bits >> (32 * mt)));
        } else {
            const uint64_t own = seen<TN>(keys, first_of(s), bits, token);
            if (__all(own == WHOLE)) return;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const uint32_t which = (uint32_t)(own >> (32 * mt)) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r) to[mt][r] = which >> (8 * (r / 4) + r % 4) & 1 ? to[mt][r] : -INFINITY;
            }
        }
    };
    uint64_t any = 0;                                   // MODE_MASK: whether a key counts
    auto put_keys = [&](uint32_t s) {
        sk.store(k_tile(s), thread);
        if (MODE == MODE_MASK) any |= sk.which;
        if (MODE == MODE_MASK && thread < TN) bias[wk][NB == 2 ? s & 1 : 0][MODE == MODE_MASK ? thread : 0] = sk.bias;
    };
    auto maximum = [&](const f32x16 (&of)[MT]) {
        float m = of[0][0];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 16; ++r) m = __builtin_elementwise_maximum(m, of[mt][r]);
        return m;
    };
    // The sum may be taken against any mark near the maximum.  A mark that is kept until a row outgrows it by 2^8 spares scaling
    // 16 DP / 32 accumulators a tile; 32-bit sums hold 2^8 times as much, and so do probabilities in 16 bits.  In float16 the mark
    // lies 2^7 below the maximum, probabilities up to 2^15 above it: one of 2^-32 of the row's largest is then rounded as one of 2^-25 would be, below
    // which float16 holds nothing.
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

    auto exponentials = [&](f32x16 (&now)[MT], typename T::V8 (&p)[MT][2][1]) {
        const float off = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) now[mt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(now[mt][r], a.scale_log2, -off));
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += now[mt][r];
            total += sum;
            p[mt][0][0] = rounded<T>(now[mt], 0);
            p[mt][1][0] = rounded<T>(now[mt], 1);
        }
    };
    auto values = [&](uint32_t s, const typename T::V8 (&p)[MT][2][1]) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int part = 0; part < 2; ++part) columns_times<T, DP, 1>(sums, v_tile(s), 32 * mt + 16 * part, p[mt][part]);
    };

    if (WR < 4) {
        // Few rows: bound by memory and by latencies, tile after tile, the next one on its way.
        if (count) {
            info[0] = info_of(0);
            sk.load(keys, a.k, a.ks, thread, first_of(0), info[0]);
            sv.load(keys, a.v, a.vs, thread, first_of(0), info[0]);
            info[1] = info_of(1);
        }
#pragma unroll 1
        for (uint32_t s = 0; s < count; ++s) {
            if (s) sync();
            put_keys(s);
            sv.store(v_tile(s), thread);
            sync();
            if (s + 1 < count) {
                sk.load(keys, a.k, a.ks, thread, first_of(s + 1), info[1]);
                sv.load(keys, a.v, a.vs, thread, first_of(s + 1), info[1]);
            }
            typename T::V8 p[MT][2][1];
            scores(x, s);
            mask(x, s);
            most = maximum(x);
            raise();
            exponentials(x, p);
            values(s, p);
            info[0] = info[1];
            info[1] = info_of(s + 2);
        }
    } else if (count) {
        // Many rows: tile s + 1's scores are formed beside tile s's exponentials, and its maximum beside tile s's product with V, so
        // that matrix and vector instructions of one wave overlap: K runs a tile ahead of V.
        f32x16 ahead[MT];
        info[0] = info_of(0);
        sk.load(keys, a.k, a.ks, thread, first_of(0), info[0]);
        sv.load(keys, a.v, a.vs, thread, first_of(0), info[0]);
        info[1] = info_of(1);
        put_keys(0);
        sv.store(v_tile(0), thread);
        sync();
        sk.load(keys, a.k, a.ks, thread, first_of(1), info[1]);
        sv.load(keys, a.v, a.vs, thread, first_of(1), info[1]);
        info[2] = info_of(2);
        scores(x, 0);
        mask(x, 0);
        most = maximum(x);
        raise();
        put_keys(1);
        sync();
        sk.load(keys, a.k, a.ks, thread, first_of(2), info[2]);
        info[0] = info[1];
        info[1] = info[2];
        info[2] = info_of(3);

        // Tile s from its scores `now`; unless it is the last, the next one's scores into `next`.
        auto step = [&](uint32_t s, f32x16 (&now)[MT], f32x16 (&next)[MT], auto more, auto masked) {
            typename T::V8 p[MT][2][1];
            constexpr int PRODUCTS = MT * DP / 16;
            if (more) scores(next, s + 1);
            exponentials(now, p);
            if (more) {
                // in one block of straight-line code: a product after every operand read and a share of the exponentials' work
                asm volatile("" ::"v"(total));
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int part = 0; part < 2; ++part) asm volatile("" ::"v"(p[mt][part][0]));
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
                for (int i = 0; i < PRODUCTS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, (MT * 56 + PRODUCTS - 1) / PRODUCTS, 0);
                }
                if (masked) mask(next, s + 1);
            }
            values(s, p);
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
            put_keys(s);
            sv.store(v_tile(s + 1), thread);
            sync();
            sk.load(keys, a.k, a.ks, thread, first_of(s + 3), info[2]);
            sv.load(keys, a.v, a.vs, thread, first_of(s + 2), info[1]);
            info[0] = info[1];
            info[1] = info[2];
            info[2] = info_of(s + 4);
        };
        // Tiles s + 1 and s + 2 are seen whole by every row: without lengths in the way all but the last, of a tree those before the nodes
        // (as far as pages are there; rows without a node are emptied at the end).
        auto whole = [&](uint32_t s) {
            return s + 3 < count && (MODE != MODE_TREE || (first_of(s + 3) <= keys.held && __all(info[0] >= 0) && __all(info[1] >= 0)));
        };
        uint32_t s = 0;
        for (; whole(s); s += 2) {
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
    // Rows without a node: tiles seen whole were not masked for them, and a probability of 0 does not clear what is infinite or NaN.
    // Rows over masked keys alone: their queries may be anything, and what is infinite or NaN in them no bias masks.
    if ((MODE == MODE_TREE && token >= keys.nodes) || (MODE == MODE_MASK && !any)) {
        top = -INFINITY;
        total = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt) o[dt] = f32x16{};
    }

    const int64_t part_row = ((int64_t)slot * a.kv_heads + kvh) * a.rows;
    if (WK == 1) {
        if (!live) return;
        const float times = total != 0.0f ? 1.0f / total : 0.0f, sum2 = total != 0.0f ? top + __log2f(total) : -INFINITY;
        if (pieces == 1) {
            store_row<T, DP>(a.o + row_at(a, a.os, b, kvh, row), o, times, a.head_dim);
            if (a.lse && h == 0) a.lse[lse_at(a, b, kvh, row)] = sum2 * LN2;
        } else {
            store_part<DP>(a.part_o + (part_row + row) * DP, o, times);
            if (h == 0) a.part_lse[part_row + row] = sum2;
        }
        return;
    }
    // Join the groups: accumulators through the tiles' memory, chunks of four values spread over the banks.
    constexpr int C4 = DP / 4, ALL = 64 * WR * WK, PER_ROW = ALL / (32 * WR);
    __syncthreads();
    f32x4 *acc = reinterpret_cast<f32x4 *>(memory);
    const int my_row = wr * 32 + n;
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const f32x4 x = {o[dt][4 * u], o[dt][4 * u + 1], o[dt][4 * u + 2], o[dt][4 * u + 3]};
            acc[(wk * 32 * WR + my_row) * C4 + ((8 * dt + 2 * u + h) ^ (n & (C4 - 1)))] = x;
        }
    if (h == 0) {
        marks[0][wk][WK > 1 ? my_row : 0] = top;
        marks[1][wk][WK > 1 ? my_row : 0] = total;
    }
    __syncthreads();
    const int r = threadIdx.x / PER_ROW, sub = threadIdx.x % PER_ROW;
    const uint32_t out_row = rt * WR * 32 + r;
    if (out_row >= a.rows) return;
    float high = -INFINITY, sum = 0.0f, weight[WK];
#pragma unroll
    for (int g = 0; g < WK; ++g) high = __builtin_elementwise_maximum(high, marks[0][g][r]);
#pragma unroll
    for (int g = 0; g < WK; ++g) {
        weight[g] = marks[0][g][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(marks[0][g][r] - high);
        sum += weight[g] * marks[1][g][r];
    }
    const float times = sum != 0.0f ? 1.0f / sum : 0.0f, sum2 = sum != 0.0f ? high + __log2f(sum) : -INFINITY;
    uint16_t *to = a.o + (pieces == 1 ? row_at(a, a.os, b, kvh, out_row) : 0);
    float *part = a.part_o + (part_row + out_row) * DP;
#pragma unroll
    for (int c = sub; c < C4; c += PER_ROW) {
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < WK; ++g) x += acc[(g * 32 * WR + r) * C4 + (c ^ (r & 31 & (C4 - 1)))] * weight[g];
        x *= times;
        if (pieces == 1) {
            if (4 * c < (int)a.head_dim) *reinterpret_cast<typename T::V4 *>(to + 4 * c) = __builtin_convertvector(x, typename T::V4);
        } else {
            *reinterpret_cast<f32x4 *>(part + 4 * c) = x;
        }
    }
    if (sub == 0) {
        if (pieces > 1) a.part_lse[part_row + out_row] = sum2;
        else if (a.lse) a.lse[lse_at(a, b, kvh, out_row)] = sum2 * LN2;
    }
}

// Joins the pieces' results: O = sum_s 2^(lse_s - max) O_s / sum_s 2^(lse_s - max), pieces in ascending order.  DP / 4 threads a row, 16 bytes each.
// Bound by memory: 32 256 rows of 128 in two pieces, 33 MB and 8 MB of results, 9.6 us, 4.3 TB/s.  In 32 bits, so that cutting costs no precision.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs a)
{
    constexpr int C4 = DP / 4, ROWS = 256 / C4;
    const int64_t all = (int64_t)a.batch * a.kv_heads * a.rows, at = (int64_t)blockIdx.x * ROWS + threadIdx.x / C4;
    const int c = threadIdx.x % C4;
    if (at >= all) return;
    const uint32_t row = (uint32_t)(at % a.rows), kvh = (uint32_t)(at / a.rows % a.kv_heads), b = (uint32_t)(at / a.rows / a.kv_heads);
    const uint32_t pieces = a.balanced ? a.cut[2 * b] : a.splits, slot = a.balanced ? a.cut[2 * b + 1] : b * a.splits;
    if (pieces == 1) return;
    const float *lse = a.part_lse + ((int64_t)slot * a.kv_heads + kvh) * a.rows + row;
    const float *part = a.part_o + (((int64_t)slot * a.kv_heads + kvh) * a.rows + row) * DP + 4 * c;
    const int64_t next = (int64_t)a.kv_heads * a.rows;
    float high = -INFINITY, sum = 0.0f;
    for (uint32_t s = 0; s < pieces; ++s) high = __builtin_elementwise_maximum(high, lse[s * next]);
    const float off = high == -INFINITY ? 0.0f : high;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t s = 0; s < pieces; ++s) {
        const float w = __builtin_amdgcn_exp2f(lse[s * next] - off);
        sum += w;
        x += *reinterpret_cast<const f32x4 *>(part + s * next * DP) * w;
    }
    x *= sum != 0.0f ? 1.0f / sum : 0.0f;
    if (4 * c < (int)a.head_dim) *reinterpret_cast<typename T::V4 *>(a.o + row_at(a, a.os, b, kvh, row) + 4 * c) = __builtin_convertvector(x, typename T::V4);
    if (a.lse && c == 0) a.lse[lse_at(a, b, kvh, row)] = sum != 0.0f ? (high + __log2f(sum)) * LN2 : -INFINITY;
}

// Gradients through float16.  Probabilities over many keys, and dS with small gradients of O, lie below the type's normal numbers (6e-5),
// where rounding is no longer relative (7e-3 of dK with gradients of 5e-4 over 2048 keys).  So P is multiplied by 2^15, and dS by a power of two of
// the lane's own (a row's in dQ, a key's in dK) that keeps it below 2^15; both are divided out of the 32-bit sums at the end.  The power starts high and
// is lowered, with the sums so far, when a value outgrows it.  It costs 3 % of dQ's time and 8 % of dK's; bfloat16, with the range of 32 bits,
// needs none of it.
constexpr float UP = 15.0f, HIGHEST = 60.0f;            // powers of two: of P; dS's over P's at first

// Keeps 16 scaled values of dS in range; returns the power of two (none or negative) that they and `sums` were multiplied by.
template <int N>
__device__ __forceinline__ float keep_in_range(f32x16 &ds, f32x16 (&sums)[N])
{
    float most = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(ds[r]));
    if (!__any(most > 0x1p15f)) return 0.0f;
    most = max_of_halves(most);
    const int lower = most > 0x1p15f ? 11 - __builtin_amdgcn_frexp_expf(most) : 0;       // to 2^10 .. 2^11
    const float by = __builtin_ldexpf(1.0f, lower);
    ds *= by;
#pragma unroll
    for (int i = 0; i < N; ++i) sums[i] *= by;
    return (float)lower;
}

// dQ, and D on the way.  As the forward pass with W waves on a tile: per tile three products, S^T = K Q^T, dP^T = V dO^T and
// dQ^T += K^T dS^T.  Split over the keys, the pieces leave their dQ in 32 bits and k_attn_sum adds them in order.
// D comes from O as it was rounded to 16 bits, the only form of it that a caller has to keep: with few keys dQ and dK are then up to 1.7 times
// as far from 64-bit values as one rounding takes them, with many 1.4 times (2-norm, bfloat16: 0.0029, 0.0024 and 0.0017).
// Nothing is added atomically, so results repeat to the bit; the price is that S and dP are formed here and again for dK and dV: seven
// products where five would do.  Bound as the forward pass is, with two thirds of the exponentials a product: 2 x 2048 rows over 4096 keys, 32 heads of 128
// over 8: 376 to 392 us, 1.07 PFLOP/s; masked, 8 x 509 over 1500, 12 heads of 64: 57 to 60 us.  Four waves with a mask over 128 values a head in
// float16 spill 2 registers, the others none.
template <class T, int DP, int W, int MODE>
__global__ __launch_bounds__(64 * W, 2) void k_attn_dq(const AttnArgs a)
{
    constexpr int TN = 64, CH = DP / 8;
    __shared__ u32x4 tiles[2][2][TN * CH];
    __shared__ __align__(16) float bias[2][MODE == MODE_MASK ? TN : 4];
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63, n = lane & 31, h = lane >> 5;
    uint32_t at = by_die(blockIdx.x, gridDim.x);
    const uint32_t rt = at % a.row_tiles;
    at /= a.row_tiles;
    const uint32_t split = at % a.splits;
    at /= a.splits;
    const uint32_t kvh = at % a.kv_heads, b = at / a.kv_heads;
    const Keys<MODE> keys(a, b, kvh);
    const uint32_t steps = (keys.end + TN - 1) / TN, per = (steps + a.splits - 1) / a.splits;
    const uint32_t step0 = split * per < steps ? split * per : steps, count = step0 + per < steps ? per : steps - step0;

    const uint32_t row = (rt * W + wave) * 32 + n;
    const bool live = row < a.rows;
    const int64_t bh = (int64_t)b * a.kv_heads + kvh;
    typename T::V8 q[DP / 16], d_o[DP / 16];
    row_operands<T, DP>(q, a.q + (live ? row_at(a, a.qs, b, kvh, row) : 0), live, a.head_dim);
    row_operands<T, DP>(d_o, a.d_o + (live ? row_at(a, a.dos, b, kvh, row) : 0), live, a.head_dim);
    float lse2 = INFINITY, delta = 0.0f;                // rows that see nothing: probabilities 0
    if (live) {
        const float l = a.lse_in[lse_at(a, b, kvh, row)];
        lse2 = l == -INFINITY ? INFINITY : l * LOG2E - (NARROW<T> ? UP + HIGHEST : 0.0f);
    }
    {
        typename T::V8 o[DP / 16];
        row_operands<T, DP>(o, a.o_in + (live ? row_at(a, a.os, b, kvh, row) : 0), live, a.head_dim);
#pragma unroll
        for (int t = 0; t < DP / 16; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta += (float)o[t][j] * (float)d_o[t][j];
        delta = sum_of_halves(delta);
        if (live && h == 0 && split == 0) a.delta[bh * a.rows + row] = delta;
    }

    f32x16 dq[1][DP / 32] = {};
    float lowered = 0.0f;                               // of dS's power of two, which lse2 holds
    Stage<DP, TN, 64 * W, MODE> sk, sv;
    auto first_of = [&](uint32_t s) { return (step0 + s) * TN; };
    auto info_of = [&](uint32_t s) { return keys.info(first_of(s) + lane); };
    int info = 0, next_info = 0;
    if (count) {
        info = info_of(0);
        sk.load(keys, a.k, a.ks, thread, first_of(0), info);
        sv.load(keys, a.v, a.vs, thread, first_of(0), info);
        next_info = info_of(1);
    }
    for (uint32_t s = 0; s < count; ++s) {
        u32x4 *kt = tiles[s & 1][0], *vt = tiles[s & 1][1];
        sk.store(kt, thread);
        sv.store(vt, thread);
        if (MODE == MODE_MASK && thread < TN) bias[s & 1][MODE == MODE_MASK ? thread : 0] = sk.bias;
        const uint64_t bits = counted<MODE, TN>(keys, first_of(s), info);
        __syncthreads();
        if (s + 1 < count) {
            info = next_info;
            sk.load(keys, a.k, a.ks, thread, first_of(s + 1), info);
            sv.load(keys, a.v, a.vs, thread, first_of(s + 1), info);
            next_info = info_of(s + 2);
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            f32x16 x = keys_by_rows<T, DP>(kt, 32 * mt, q, MODE == MODE_MASK ? biases(bias[s & 1] + (MODE == MODE_MASK ? 32 * mt : 0)) : f32x16{});
            const f32x16 dp = keys_by_rows<T, DP>(vt, 32 * mt, d_o);
            if (MODE == MODE_PLAIN && bits != ~0ull) mask_keys(x, (uint32_t)(bits >> (32 * mt)));
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
    if (MODE == MODE_MASK && lse2 == INFINITY) {        // (a row that sees nothing, whatever its query holds)
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt) dq[0][dt] = f32x16{};
    }
    const float times = NARROW<T> ? a.scale * __builtin_amdgcn_exp2f(-(UP + HIGHEST + lowered)) : a.scale;
    if (a.splits == 1) store_row<T, DP>(a.dq + row_at(a, a.dqs, b, kvh, row), dq[0], times, a.head_dim);
    else store_part<DP>(a.part_o + (((int64_t)split * a.batch * a.kv_heads + bh) * a.rows + row) * DP, dq[0], times);
}

// dK and dV of 32 W keys, 32 a wave, over the rows of a piece, TR of them between two barriers.  Per 32 rows: S = Q K^T, dP = dO V^T
// (rows along m, a lane holds one key), dV^T += dO^T P, dK^T += Q^T dS; the rows' Q and dO are read from shared memory both along and across.
// With 128 values a head the 256 registers of a wave hold K and both sums; V's operands lie in shared memory (their reads are what
// limits it most), with 32 rows a step: 64 spilled 67 registers and took 900 us.  2 x 2048 rows over 4096 keys, 32 heads of 128 over 8: 510 to
// 540 us, 1.05 PFLOP/s; masked, 8 x 509 over 1500, 12 heads of 64: 65 to 69 us.  With four waves 10 registers are spilled in bfloat16 and 18 in
// float16 (some of them read again in the loop), with eight none and 8.
template <class T, int DP, int W, int MODE>
__global__ __launch_bounds__(64 * W, 2) void k_attn_dkv(const AttnArgs a)
{
    constexpr int TR = DP == 128 ? 32 : 64, CH = DP / 8, LOADS = TR * CH / (64 * W), ROWS = 64 * W / CH;
    static_assert(LOADS * 64 * W == TR * CH && 2 * TR <= 64 * W, "a tile is dealt out evenly, its statistics to two threads a row");
    __shared__ u32x4 tiles[2][2][TR * CH];
    __shared__ f32x4 stats[2][2][TR / 4];               // lse in powers of two, D
    constexpr bool AWAY = DP == 128;                    // V's operands in shared memory: with them 256 registers do not suffice
    __shared__ u32x4 away[AWAY ? W : 1][DP / 16][64];
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63, n = lane & 31, h = lane >> 5;
    const uint32_t key_tiles = (a.kv_len + 32 * W - 1) / (32 * W);
    uint32_t at = by_die(blockIdx.x, gridDim.x);
    const uint32_t kt = at % key_tiles;
    at /= key_tiles;
    const uint32_t split = at % a.splits;
    at /= a.splits;
    const uint32_t kvh = at % a.kv_heads, b = at / a.kv_heads;
    const Keys<MODE> keys(a, b, kvh);
    const uint32_t key = (kt * W + wave) * 32 + n;
    const uint32_t steps = kt * 32 * W < keys.end ? (a.rows + TR - 1) / TR : 0, per = (steps + a.splits - 1) / a.splits;
    const uint32_t step0 = split * per < steps ? split * per : steps, count = step0 + per < steps ? per : steps - step0;

    const bool valid = key < keys.end && keys.info(key) >= 0;
    typename T::V8 k[DP / 16], v[DP / 16];
    row_operands<T, DP>(k, a.k + (valid ? b * a.ks.batch + key * a.ks.token + kvh * a.ks.head : 0), valid, a.head_dim);
    row_operands<T, DP>(v, a.v + (valid ? b * a.vs.batch + key * a.vs.token + kvh * a.vs.head : 0), valid, a.head_dim);
    if (AWAY) {                                         // a lane reads what it has written itself
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) away[AWAY ? wave : 0][t][lane] = __builtin_bit_cast(u32x4, v[t]);
    }
    const int64_t bh = (int64_t)b * a.kv_heads + kvh;

    // Rows past the last one repeat its Q, and their dO is zeros, as their probabilities do not clear an infinite gradient.  Columns past the
    // head's repeat the first ones: K and V are 0 there.
    u32x4 rq[LOADS], ro[LOADS];
    float stat = 0.0f;
    const int row0 = thread / CH, c = 8 * (thread % CH) < (int)a.head_dim ? thread % CH : 0;
    auto load = [&](uint32_t s) {
        const uint32_t first = (step0 + s) * TR;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t row = first + row0 + i * ROWS, token = token_of(a, row < a.rows ? row : a.rows - 1), head = kvh * a.group + ((row < a.rows ? row : a.rows - 1) - token * a.group);
            rq[i] = *reinterpret_cast<const u32x4 *>(a.q + (b * a.qs.batch + token * a.qs.token + head * a.qs.head + c * 8));
            ro[i] = zeros();
            if (row < a.rows) ro[i] = *reinterpret_cast<const u32x4 *>(a.d_o + (b * a.dos.batch + token * a.dos.token + head * a.dos.head + c * 8));
        }
        const uint32_t row = first + thread % TR;
        const bool there = row < a.rows;
        if (thread < TR) {
            const float l = a.lse_in[lse_at(a, b, kvh, there ? row : a.rows - 1)];
            stat = there && l != -INFINITY ? l * LOG2E - (NARROW<T> ? UP : 0.0f) : INFINITY;      // rows that are not there, or see nothing: probabilities 0
        } else if (thread < 2 * TR) {
            stat = a.delta[bh * a.rows + (there ? row : a.rows - 1)];
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
            qt[chunk_at<CH>(row0 + i * ROWS, thread % CH)] = rq[i];
            ot[chunk_at<CH>(row0 + i * ROWS, thread % CH)] = ro[i];
        }
        if (thread < 2 * TR) reinterpret_cast<float *>(stats[s & 1])[thread] = stat;
        __syncthreads();
        if (s + 1 < count) load(s + 1);
#pragma unroll
        for (int sub = 0; sub < TR / 32; ++sub) {
            f32x16 x = {}, dp = {};
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) x = T::mma(as_operand<T>(qt[32 * sub * CH + chunk_at<CH>(n, 2 * t + h)]), k[t], x);
#pragma unroll
            for (int t = 0; t < DP / 16; ++t)
                dp = T::mma(as_operand<T>(ot[32 * sub * CH + chunk_at<CH>(n, 2 * t + h)]), AWAY ? as_operand<T>(away[AWAY ? wave : 0][t][lane]) : v[t], dp);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 lse2 = stats[s & 1][0][8 * sub + 2 * g + h], delta = stats[s & 1][1][8 * sub + 2 * g + h];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 4 * g + j;
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale_log2, -lse2[j]));
                    x[r] = p;
                    dp[r] = p * (NARROW<T> ? (dp[r] - delta[j]) * by : dp[r] - delta[j]);
                }
            }
            if (NARROW<T>) by *= __builtin_amdgcn_exp2f(keep_in_range(dp, dk[0]));
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const typename T::V8 p[1] = {rounded<T>(x, part)}, ds[1] = {rounded<T>(dp, part)};
                columns_times<T, DP, 1>(dv, ot, 32 * sub + 16 * part, p);
                columns_times<T, DP, 1>(dk, qt, 32 * sub + 16 * part, ds);
            }
        }
    }
    if (key >= a.kv_len) return;
    if (!valid) {                                       // (what a lane has gathered for a key that does not count)
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt) dk[0][dt] = dv[0][dt] = f32x16{};
    }
    const float times = NARROW<T> ? a.scale * 0x1p-15f / by : a.scale, times_v = NARROW<T> ? 0x1p-15f : 1.0f;
    if (a.splits == 1) {
        store_row<T, DP>(a.dk + b * a.dks.batch + key * a.dks.token + kvh * a.dks.head, dk[0], times, a.head_dim);
        store_row<T, DP>(a.dv + b * a.dvs.batch + key * a.dvs.token + kvh * a.dvs.head, dv[0], times_v, a.head_dim);
    } else {
        float *part = a.part_o + ((((int64_t)split * a.batch * a.kv_heads + bh) * a.kv_len + key) * 2) * DP;
        store_part<DP>(part, dk[0], times);
        store_part<DP>(part + DP, dv[0], times_v);
    }
}

// Sums of pieces in ascending order, rounded once: which = 0: dQ rows; 1: dK and dV of a key beside each other.  Bound by memory:
// four pieces of dK and dV of 1024 keys, 16 heads of 128, 67 MB: 13 us, 5.2 TB/s (some of it from the last level of cache).
template <class T, int DP, int WHICH>
__global__ __launch_bounds__(256) void k_attn_sum(const AttnArgs a)
{
    constexpr int C4 = DP / 4 * (WHICH + 1), LINES = 256 / C4;
    const uint32_t lines = WHICH ? a.kv_len : a.rows;
    const int64_t all = (int64_t)a.batch * a.kv_heads * lines, at = (int64_t)blockIdx.x * LINES + threadIdx.x / C4;
    const int c = threadIdx.x % C4;
    if (at >= all) return;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t s = 0; s < a.splits; ++s) x += *reinterpret_cast<const f32x4 *>(a.part_o + ((s * all + at) * C4 + c) * 4);
    const uint32_t line = (uint32_t)(at % lines), kvh = (uint32_t)(at / lines % a.kv_heads), b = (uint32_t)(at / lines / a.kv_heads);
    const int d = 4 * c % DP;
    if (d >= (int)a.head_dim) return;
    uint16_t *to;
    if (!WHICH) to = a.dq + row_at(a, a.dqs, b, kvh, line);
    else if (4 * c < DP) to = a.dk + b * a.dks.batch + line * a.dks.token + kvh * a.dks.head;
    else to = a.dv + b * a.dvs.batch + line * a.dvs.token + kvh * a.dvs.head;
    *reinterpret_cast<typename T::V4 *>(to + d) = __builtin_convertvector(x, typename T::V4);
}

}  // namespace mmee
