// Host side of the attention operators: argument checks, the choice of variant and pieces, launches.
#include <algorithm>
#include <cmath>

#include "attention.h"

namespace mmee {
namespace {

constexpr uint64_t MOST_ROWS = 1u << 28;        // rows of one key/value head, keys: token_of() and key numbers stay exact
constexpr int64_t MOST_TOKEN_STRIDE = 1 << 24;  // a tile's offsets fit 32 bits

bool misaligned(const void *p) { return ((uintptr_t)p & 15) != 0; }

// Strides of a tensor of `batch` x `tokens` x `heads` rows: 16-byte aligned rows, nothing negative; an output's rows are rows of their own.
bool take_strides(const int64_t *given, uint64_t batch, uint64_t tokens, uint64_t heads, bool output, Strides &out)
{
    const uint64_t extent[3] = {batch, tokens, heads};
    int64_t s[3];
    for (int k = 0; k < 3; ++k) {
        s[k] = extent[k] > 1 ? given[k] : 0;
        if (s[k] < 0 || s[k] % 8 || s[k] > (int64_t)1 << 46 || (output && extent[k] > 1 && s[k] == 0)) return false;
    }
    if (s[1] > MOST_TOKEN_STRIDE) return false;
    out = {s[0], s[1], s[2]};
    return true;
}

int padded(uint32_t head_dim) { return head_dim <= 32 ? 32 : head_dim <= 64 ? 64 : 128; }

struct AttnPlan {
    AttnArgs a = {};
    int dp = 0, dtype = 0, mode = MODE_PLAIN, row_waves = 4, dq_waves = 4, dkv_waves = 4;
    uint32_t blocks = 0;                        // of the forward pass
    uint32_t dq_splits = 1, dkv_splits = 1;
    uint64_t dq_blocks = 0, dkv_blocks = 0;
    bool joins = false;                         // the forward pass leaves pieces
    uint64_t part_bytes = 0, lse_bytes = 0, forward_bytes = 0, backward_bytes = 0;
};

// Whether blocks that run alone on a unit keep the card busy: more than half of the units in one round, or 7/8 in whole rounds.
bool fills(uint64_t blocks) { return blocks > 128 && (blocks <= 256 || blocks * 8 >= (blocks + 255) / 256 * 256 * 7); }

// Pieces of the keys (or rows) such that about `room` blocks run, none of them shorter than `least` steps.
uint32_t pieces(uint64_t blocks, uint64_t steps, uint64_t least, uint64_t room)
{
    if (!blocks || blocks >= room * 3 / 4) return 1;
    const uint64_t most = std::max<uint64_t>(1, steps / least);
    return (uint32_t)std::min<uint64_t>({most, std::max<uint64_t>(1, room / blocks), 128});
}

uint64_t up256(uint64_t x) { return (x + 255) & ~(uint64_t)255; }

// Tiles of 32 rows a wave and pieces of the keys, for `row_waves` waves with rows of their own; returns the number of blocks.
// Up to 32 rows the four waves of a block take tiles of keys of their own, up to 64 two do.
uint64_t split(AttnPlan &p, int row_waves, uint64_t kv_len, bool ragged)
{
    AttnArgs &a = p.a;
    const uint64_t batch = a.batch;
    a.row_tiles = (a.rows + 32 * row_waves - 1) / (32 * row_waves);
    // Blocks of four waves run two to a compute unit, of eight waves alone.  With up to 32 rows eight waves halve the number of steps, which
    // counts while there are fewer blocks than units; pieces cost a second launch that joins them: none shorter than 512 keys.
    const uint64_t each = (uint64_t)a.row_tiles * a.kv_heads, room = row_waves == 8 ? 256 : 512;
    a.step_keys = row_waves > 1 ? 64 : each * batch * std::max<uint64_t>(1, kv_len / 512) <= 256 ? 256 : 128;
    a.least = 512 / a.step_keys;
    const uint64_t steps = (kv_len + a.step_keys - 1) / a.step_keys;
    a.splits = 1;
    a.slots = a.batch;
    a.balanced = false;
    if (each && each * batch < room && steps > a.least) {         // pieces for one round of blocks (two, three and four rounds were 15 to 40 % slower)
        a.slots = (uint32_t)std::min<uint64_t>(std::max<uint64_t>(room / each, batch), batch * (steps / a.least));
        a.balanced = ragged && batch > 1 && batch <= 64 && a.slots > batch;
        if (!a.balanced) {
            a.splits = a.slots / a.batch;
            a.slots = a.splits * a.batch;
        }
    }
    return each * a.slots;
}

int common(AttnPlan &p, uint32_t dtype, uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t head_dim, uint32_t q_len, uint64_t kv_len, float scale, bool ragged)
{
    if (dtype != MMEE_F16 && dtype != MMEE_BF16) return MMEE_EINVAL;
    if (!batch || !heads || !kv_heads || heads % kv_heads || !head_dim || head_dim % 8 || head_dim > 128) return MMEE_EINVAL;
    if (!(scale > 0.0f) || !std::isfinite(scale)) return MMEE_EINVAL;
    const uint64_t group = heads / kv_heads, rows = group * q_len;
    if (rows > MOST_ROWS || group > 4096 || kv_len > MOST_ROWS || (uint64_t)batch * heads > 1u << 24) return MMEE_EINVAL;
    AttnArgs &a = p.a;
    p.dtype = (int)dtype;
    p.dp = padded(head_dim);
    a.batch = batch;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.group = (uint32_t)group;
    // r / group = r * ceil(2^shift / group) >> shift for every r < 2^32, with 2^shift >= 2^32 group; the product stays below 2^64 for r < 2^28
    a.group_shift = 32;
    while ((uint64_t)1 << (a.group_shift - 32) < group) ++a.group_shift;
    a.group_inverse = (((uint64_t)1 << a.group_shift) + group - 1) / group;
    a.q_len = q_len;
    a.rows = (uint32_t)rows;
    a.kv_len = (uint32_t)kv_len;
    a.head_dim = head_dim;
    a.scale = scale;
    a.scale_log2 = scale * LOG2E;
    // Eight waves with rows of their own read every key half as often as four, but their tiles may leave units without work.  Microseconds,
    // 256 rows against 128, rows x keys x heads, 128 a head: 4096 x 4096 x 16 139 : 156, 200 x 2048 x 128 51 : 54, 1024 x 1024 x 128 87 : 92;
    // not taken: 1024 x 1024 x 16 35 : 32, 640 x 640 x 128 56 : 50, 197 x 197 x 384 34 : 31, 256 x 512 x 128 25 : 21.
    p.row_waves = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    if (rows > 128 && p.dp >= 64) {
        const uint64_t blocks = split(p, 8, kv_len, ragged);
        if (fills(blocks)) p.row_waves = 8;
    }
    const uint64_t blocks = split(p, p.row_waves, kv_len, ragged);
    if (blocks > 0x7fffffff) return MMEE_EINVAL;
    p.blocks = (uint32_t)blocks;
    p.joins = a.slots > batch;
    p.part_bytes = up256(4ull * a.slots * kv_heads * rows * p.dp);
    p.lse_bytes = up256(4ull * a.slots * kv_heads * rows);
    p.forward_bytes = p.joins ? p.part_bytes + p.lse_bytes + (a.balanced ? up256(8 * batch) : 0) : 0;
    return MMEE_OK;
}

int plan_attn(const mmee_attn *x, bool pointers, AttnPlan &p)
{
    if (!x || x->reserved) return MMEE_EINVAL;
    const int rc = common(p, x->dtype, x->batch, x->heads, x->kv_heads, x->head_dim, x->q_len, x->kv_len, x->scale, x->kv_lens != nullptr);
    if (rc) return rc;
    AttnArgs &a = p.a;
    if (!take_strides(x->q_stride, x->batch, x->q_len, x->heads, false, a.qs) || !take_strides(x->k_stride, x->batch, x->kv_len, x->kv_heads, false, a.ks) ||
        !take_strides(x->v_stride, x->batch, x->kv_len, x->kv_heads, false, a.vs) || !take_strides(x->o_stride, x->batch, x->q_len, x->heads, true, a.os))
        return MMEE_EINVAL;
    if (x->key_mask && x->mask_stride < 0) return MMEE_EINVAL;
    p.mode = x->key_mask ? MODE_MASK : MODE_PLAIN;
    a.q = (const uint16_t *)x->q;
    a.k = (const uint16_t *)x->k;
    a.v = (const uint16_t *)x->v;
    a.o = (uint16_t *)x->o;
    a.lse = x->lse;
    a.kv_lens = x->kv_lens;
    a.key_mask = x->key_mask;
    a.mask_stride = x->batch > 1 ? x->mask_stride : 0;
    if (pointers) {
        if ((a.rows && (!x->q || !x->o)) || (x->kv_len && (!x->k || !x->v))) return MMEE_EINVAL;
        if (misaligned(x->q) || misaligned(x->k) || misaligned(x->v) || misaligned(x->o) || misaligned(x->workspace) || ((uintptr_t)x->lse & 3) || ((uintptr_t)x->kv_lens & 3))
            return MMEE_EINVAL;
    }
    // Backward.  Blocks of eight waves read rows or keys half as often as blocks of four, and run alone on a unit, so that nothing covers
    // the beginning and the end of a short one.  Microseconds, eight against four.  dQ, rows x keys x heads, 128 a head: 4096 x 4096 x 16
    // 183 : 199, 200 x 2048 x 128 64 : 70, 2048 x 4096 x 64 390 : 424; not taken: 512 x 512 x 512 146 : 139, 640 x 640 x 128 70 : 63, 64 a
    // head 1024 x 1024 x 128 67 : 64 (and 107 : 112 at 4096 x 4096 x 16).  dK and dV, 128 a head: 4096 x 4096 x 16 251 : 284,
    // 256 x 512 x 128 37 : 39, 64 a head 4096 x 4096 x 16 139 : 152; not taken: 197 x 197 x 384 49 : 47, 64 a head 200 x 2048 x 128 68 : 63.
    const uint64_t heads_all = (uint64_t)a.batch * a.kv_heads;
    uint64_t tiles = 0, key_tiles = 0;
    for (const int waves : {8, 4}) {
        tiles = ((uint64_t)a.rows + 32 * waves - 1) / (32 * waves);
        p.dq_waves = waves;
        p.dq_splits = pieces(tiles * heads_all, ((uint64_t)a.kv_len + 63) / 64, 4, 2048 / waves);
        if (p.dp == 128 && a.rows > 128 && a.kv_len / p.dq_splits >= 1024 && fills(tiles * heads_all * p.dq_splits)) break;
    }
    for (const int waves : {8, 4}) {
        key_tiles = ((uint64_t)a.kv_len + 32 * waves - 1) / (32 * waves);
        p.dkv_waves = waves;
        p.dkv_splits = pieces(key_tiles * heads_all, ((uint64_t)a.rows + 31) / 32, 8, 2048 / waves);
        if ((p.dp == 128 || (p.dp == 64 && a.rows >= 1024)) && a.kv_len > 128 && fills(key_tiles * heads_all * p.dkv_splits)) break;
    }
    p.dq_blocks = tiles * heads_all * p.dq_splits;
    p.dkv_blocks = key_tiles * heads_all * p.dkv_splits;
    if (p.dq_blocks > 0x7fffffff || p.dkv_blocks > 0x7fffffff) return MMEE_EINVAL;
    const uint64_t dq_parts = p.dq_splits > 1 ? 4 * p.dq_splits * heads_all * a.rows * p.dp : 0;
    const uint64_t dkv_parts = p.dkv_splits > 1 ? 8 * p.dkv_splits * heads_all * a.kv_len * p.dp : 0;
    p.backward_bytes = up256(4 * heads_all * a.rows) + up256(std::max(dq_parts, dkv_parts));
    return MMEE_OK;
}

int plan_tree(const mmee_tree_attn *x, bool pointers, AttnPlan &p)
{
    if (!x || x->reserved || !x->page_tokens || (x->page_tokens & (x->page_tokens - 1)) || x->page_tokens > 1u << 16 || x->nodes > 1024) return MMEE_EINVAL;
    const int rc = common(p, x->dtype, x->batch, x->heads, x->kv_heads, x->head_dim, x->nodes, (uint64_t)x->pages_per_seq * x->page_tokens, x->scale, true);
    if (rc) return rc;
    AttnArgs &a = p.a;
    p.mode = MODE_TREE;
    if (!take_strides(x->q_stride, x->batch, x->nodes, x->heads, false, a.qs) || !take_strides(x->o_stride, x->batch, x->nodes, x->heads, true, a.os) ||
        !take_strides(x->k_stride, x->n_pages, x->page_tokens, x->kv_heads, false, a.ks) ||
        !take_strides(x->v_stride, x->n_pages, x->page_tokens, x->kv_heads, false, a.vs))
        return MMEE_EINVAL;
    if (x->n_pages > 0x7fffffff || x->table_stride < 0) return MMEE_EINVAL;
    a.q = (const uint16_t *)x->q;
    a.k = (const uint16_t *)x->k_pages;
    a.v = (const uint16_t *)x->v_pages;
    a.o = (uint16_t *)x->o;
    a.lse = x->lse;
    a.page_table = x->page_table;
    a.table_stride = x->batch > 1 ? x->table_stride : 0;
    a.cache_lens = x->cache_lens;
    a.node_counts = x->node_counts;
    a.ancestors = x->ancestors;
    a.words = (x->nodes + 63) / 64;
    a.n_pages = x->n_pages;
    while ((1u << a.page_shift) < x->page_tokens) ++a.page_shift;
    if (pointers) {
        if (a.rows && (!x->q || !x->o || !x->cache_lens || !x->ancestors)) return MMEE_EINVAL;
        if ((x->n_pages && (!x->k_pages || !x->v_pages)) || (a.kv_len && !x->page_table)) return MMEE_EINVAL;
        if (misaligned(x->q) || misaligned(x->k_pages) || misaligned(x->v_pages) || misaligned(x->o) || misaligned(x->workspace) || ((uintptr_t)x->ancestors & 7) ||
            (((uintptr_t)x->lse | (uintptr_t)x->page_table | (uintptr_t)x->cache_lens | (uintptr_t)x->node_counts) & 3))
            return MMEE_EINVAL;
    }
    return MMEE_OK;
}

template <class T, int DP, int MODE>
void forward_as(const AttnPlan &p, Launching &l)
{
    if (p.row_waves == 8) {
        if constexpr (DP >= 64) l.run(k_attn_forward<T, DP, 8, 1, MODE>, p.blocks, 512, p.a);
    } else if (p.row_waves == 4) l.run(k_attn_forward<T, DP, 4, 1, MODE>, p.blocks, 256, p.a);
    else if (p.row_waves == 2) l.run(k_attn_forward<T, DP, 2, 2, MODE>, p.blocks, 256, p.a);
    else if (p.a.step_keys == 128) l.run(k_attn_forward<T, DP, 1, 4, MODE>, p.blocks, 256, p.a);
    else l.run(k_attn_forward<T, DP, 1, 8, MODE>, p.blocks, 512, p.a);
    if (p.joins) {
        const uint64_t lines = (uint64_t)p.a.batch * p.a.kv_heads * p.a.rows, per = 256 / (DP / 4);
        l.run(k_attn_join<T, DP>, (lines + per - 1) / per, 256, p.a);
    }
}

template <class T, int DP, int MODE>
void backward_as(const AttnPlan &p, Launching &l)
{
    const uint64_t heads_all = (uint64_t)p.a.batch * p.a.kv_heads;
    AttnArgs a = p.a;
    if (p.dq_blocks) {
        a.row_tiles = (a.rows + 32 * p.dq_waves - 1) / (32 * p.dq_waves);
        a.splits = p.dq_splits;
        if (p.dq_waves == 8) {
            if constexpr (DP == 128) l.run(k_attn_dq<T, DP, 8, MODE>, p.dq_blocks, 512, a);
        } else {
            l.run(k_attn_dq<T, DP, 4, MODE>, p.dq_blocks, 256, a);
        }
        const uint64_t per = 256 / (DP / 4);
        if (a.splits > 1) l.run(k_attn_sum<T, DP, 0>, (heads_all * a.rows + per - 1) / per, 256, a);
    }
    if (p.dkv_blocks) {
        a.splits = p.dkv_splits;
        if (p.dkv_waves == 8) {
            if constexpr (DP >= 64) l.run(k_attn_dkv<T, DP, 8, MODE>, p.dkv_blocks, 512, a);
        } else {
            l.run(k_attn_dkv<T, DP, 4, MODE>, p.dkv_blocks, 256, a);
        }
        const uint64_t per = 256 / (DP / 2);
        if (a.splits > 1) l.run(k_attn_sum<T, DP, 1>, (heads_all * a.kv_len + per - 1) / per, 256, a);
    }
}

// Calls f.template run<T, DP, MODE>() for the plan's type, padded head size and mode.
template <class F>
void dispatch(const AttnPlan &p, F f)
{
    auto with_mode = [&](auto type, auto dp) {
        if (p.mode == MODE_PLAIN) f(type, dp, std::integral_constant<int, MODE_PLAIN>());
        else if (p.mode == MODE_MASK) f(type, dp, std::integral_constant<int, MODE_MASK>());
        else f(type, dp, std::integral_constant<int, MODE_TREE>());
    };
    auto with_dp = [&](auto type) {
        if (p.dp == 32) with_mode(type, std::integral_constant<int, 32>());
        else if (p.dp == 64) with_mode(type, std::integral_constant<int, 64>());
        else with_mode(type, std::integral_constant<int, 128>());
    };
    if (p.dtype == MMEE_F16) with_dp(F16());
    else with_dp(BF16());
}

int forward(AttnPlan &p, void *workspace, uint64_t workspace_bytes)
{
    if (p.forward_bytes && (!workspace || workspace_bytes < p.forward_bytes)) return MMEE_EWORKSPACE;
    if (!p.blocks) return MMEE_OK;
    p.a.part_o = (float *)workspace;
    p.a.part_lse = p.a.part_o + p.part_bytes / 4;
    p.a.cut = (uint32_t *)(p.a.part_lse + p.lse_bytes / 4);
    Launching l;
    if (l.rc) return l.rc;
    dispatch(p, [&](auto type, auto dp, auto mode) { forward_as<decltype(type), dp.value, mode.value>(p, l); });
    return l.result("attention, forward");
}

}  // namespace
}  // namespace mmee

using namespace mmee;

extern "C" {

int mmee_attn_workspace(const mmee_attn *x, int backward, uint64_t *bytes)
{
    if (!bytes) return MMEE_EINVAL;
    if (!x) return MMEE_EINVAL;
    // enough with and without lengths, which decide how the keys are cut: they may be given later
    *bytes = 0;
    static const int32_t some = 0;
    for (const int32_t *lens : {(const int32_t *)nullptr, &some}) {
        mmee_attn y = *x;
        y.kv_lens = lens;
        AttnPlan p;
        const int rc = plan_attn(&y, false, p);
        if (rc) return rc;
        *bytes = std::max({*bytes, p.forward_bytes, backward ? p.backward_bytes : 0});
    }
    return MMEE_OK;
}

int mmee_attn_forward(const mmee_attn *x)
{
    AttnPlan p;
    const int rc = plan_attn(x, true, p);
    return rc ? rc : forward(p, x->workspace, x->workspace_bytes);
}

int mmee_attn_backward(const mmee_attn *x, const mmee_attn_grads *g)
{
    AttnPlan p;
    const int rc = plan_attn(x, true, p);
    if (rc) return rc;
    AttnArgs &a = p.a;
    if (!g || (a.rows && (!x->lse || !g->d_o || !g->dq)) || (a.kv_len && (!g->dk || !g->dv))) return MMEE_EINVAL;
    if (misaligned(g->d_o) || misaligned(g->dq) || misaligned(g->dk) || misaligned(g->dv)) return MMEE_EINVAL;
    if (!take_strides(g->do_stride, a.batch, a.q_len, a.heads, false, a.dos) || !take_strides(g->dq_stride, a.batch, a.q_len, a.heads, true, a.dqs) ||
        !take_strides(g->dk_stride, a.batch, a.kv_len, a.kv_heads, true, a.dks) || !take_strides(g->dv_stride, a.batch, a.kv_len, a.kv_heads, true, a.dvs))
        return MMEE_EINVAL;
    if (p.backward_bytes && (!x->workspace || x->workspace_bytes < p.backward_bytes)) return MMEE_EWORKSPACE;
    if (!p.dq_blocks && !p.dkv_blocks) return MMEE_OK;
    a.o_in = (const uint16_t *)x->o;
    a.lse_in = x->lse;
    a.d_o = (const uint16_t *)g->d_o;
    a.dq = (uint16_t *)g->dq;
    a.dk = (uint16_t *)g->dk;
    a.dv = (uint16_t *)g->dv;
    a.delta = (float *)x->workspace;
    a.part_o = a.delta + up256(4ull * a.batch * a.kv_heads * a.rows) / 4;
    Launching l;
    if (l.rc) return l.rc;
    dispatch(p, [&](auto type, auto dp, auto mode) {
        if constexpr (mode.value != MODE_TREE) backward_as<decltype(type), dp.value, mode.value>(p, l);
    });
    return l.result("attention, backward");
}

int mmee_tree_attn_workspace(const mmee_tree_attn *x, uint64_t *bytes)
{
    if (!bytes) return MMEE_EINVAL;
    AttnPlan p;
    const int rc = plan_tree(x, false, p);
    if (rc) return rc;
    *bytes = p.forward_bytes;
    return MMEE_OK;
}

int mmee_tree_attn_forward(const mmee_tree_attn *x)
{
    AttnPlan p;
    const int rc = plan_tree(x, true, p);
    return rc ? rc : forward(p, x->workspace, x->workspace_bytes);
}

}  // extern "C"
