// Host side of the norm and rotation of queries and keys and of appending to a paged cache: argument checks, the choice of variant, launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "rotate.h"

namespace mmee {
namespace {

constexpr uint32_t MOST_TOKENS = (1u << 26) - 4;       // a wave each: a launch has less than 2^32 threads

bool misaligned(std::initializer_list<const void *> list, uintptr_t to)
{
    for (const void *p : list)
        if ((uintptr_t)p & (to - 1)) return true;
    return false;
}

// A stride in elements: rows that are 16-byte aligned, nothing negative, an output's rows their own; not looked at where there is one row.
bool take(int64_t given, uint64_t extent, bool output, int64_t &to)
{
    to = extent > 1 ? given : 0;
    return to >= 0 && to % 8 == 0 && to <= (int64_t)1 << 46 && !(output && extent > 1 && to == 0);
}

bool take(const int64_t *given, uint64_t tokens, uint64_t heads, bool output, Rows &to)
{
    return take(given[0], tokens, output, to.token) && take(given[1], heads, output, to.head);
}

// An output in its input's place has to lie as the input does.
bool moved(const void *in, const Rows &at, const void *out, const Rows &to) { return in && in == out && (at.token != to.token || at.head != to.head); }

// Waves that share a token's heads: one, unless that leaves the card without work.  A wave on its own works the angles out once for all heads.
uint32_t shares(uint64_t tokens, uint64_t heads, uint32_t lanes)
{
    const uint64_t most = (heads * lanes + 63) / 64;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(most, 4096 / std::max<uint64_t>(tokens, 1)));
}

uint32_t lanes_of(uint32_t head_dim) { return head_dim <= 32 ? 2 : head_dim <= 64 ? 4 : head_dim <= 128 ? 8 : 16; }

// What the two structures have in common.
template <class X>
int common(const X *x, RotateArgs &r)
{
    if ((x->dtype != MMEE_F16 && x->dtype != MMEE_BF16) || x->pairs > MMEE_PAIRS_NEIGHBOURS) return MMEE_EINVAL;
    if (!x->head_dim || x->head_dim % 8 || x->head_dim > 256 || x->rot_dim % 16 || x->rot_dim > x->head_dim) return MMEE_EINVAL;
    if (x->tokens > MOST_TOKENS || x->heads > 1u << 16 || x->kv_heads > 1u << 16 || !x->axes || x->axes > 4 || x->axis_stride < 0) return MMEE_EINVAL;
    r.tokens = x->tokens;
    r.heads = x->heads;
    r.kv_heads = x->kv_heads;
    r.head_dim = x->head_dim;
    r.rot = x->rot_dim;
    r.axes = x->axes;
    r.eps = x->eps;
    r.q = (const uint16_t *)x->q;
    r.k = (const uint16_t *)x->k;
    r.q_weight = (const uint16_t *)x->q_weight;
    r.k_weight = (const uint16_t *)x->k_weight;
    r.freqs = x->freqs;
    r.positions = x->rot_dim ? x->positions : nullptr;
    r.axis_stride = x->axes > 1 ? x->axis_stride : 0;
    r.axis_of = x->rot_dim ? x->axis_of : nullptr;
    if ((x->q_weight || x->k_weight) && !(x->eps >= 1e-30f && std::isfinite(x->eps))) return MMEE_EINVAL;
    if (misaligned({x->q, x->k, x->q_weight, x->k_weight, x->q_out}, 16) || misaligned({x->freqs}, 8) || misaligned({x->positions}, 4)) return MMEE_EINVAL;
    if (x->rot_dim && x->tokens && !x->freqs) return MMEE_EINVAL;
    return MMEE_OK;
}

int plan_rotate(const mmee_qk_rotate *x, bool pointers, RotateArgs &r)
{
    if (!x || x->reserved || !x->heads || !x->kv_heads) return MMEE_EINVAL;
    mmee_qk_rotate y = *x;
    if (!pointers) {                            // (only their being there matters)
        static const double some = 0;
        y.freqs = &some;
        y.positions = nullptr;
        y.q = y.k = y.q_out = y.k_out = nullptr;
    }
    const int rc = common(&y, r);
    if (rc) return rc;
    if (!x->q_weight != !x->k_weight) return MMEE_EINVAL;
    if (!take(x->q_stride, r.tokens, r.heads, false, r.qs) || !take(x->k_stride, r.tokens, r.kv_heads, false, r.ks) || !take(x->q_out_stride, r.tokens, r.heads, true, r.qos) ||
        !take(x->k_out_stride, r.tokens, r.kv_heads, true, r.kos))
        return MMEE_EINVAL;
    r.q_out = (uint16_t *)x->q_out;
    r.k_out = (uint16_t *)x->k_out;
    if (pointers && (moved(x->q, r.qs, x->q_out, r.qos) || moved(x->k, r.ks, x->k_out, r.kos))) return MMEE_EINVAL;
    if (pointers && r.tokens && (!x->q || !x->k || !x->q_out || !x->k_out || (r.rot && !x->positions) || misaligned({x->k_out, x->workspace}, 16))) return MMEE_EINVAL;
    r.shares = shares(r.tokens, r.heads + r.kv_heads, lanes_of(r.head_dim));
    // Backward: blocks whose lines of the weights' gradients stay few, four to a unit, as many as run at once.
    r.blocks = (uint32_t)std::min<uint64_t>(((uint64_t)r.tokens * r.shares + 3) / 4, 1024);
    return MMEE_OK;
}

uint64_t parts_bytes(const RotateArgs &r) { return r.q_weight ? 8ull * r.blocks * r.head_dim : 0; }

// Calls f(type, lanes of a head, neighbours).
template <class F>
void dispatch(uint32_t dtype, uint32_t pairs, uint32_t head_dim, F f)
{
    auto with_lanes = [&](auto type, auto near) {
        switch (lanes_of(head_dim)) {
        case 2: return f(type, std::integral_constant<int, 2>(), near);
        case 4: return f(type, std::integral_constant<int, 4>(), near);
        case 8: return f(type, std::integral_constant<int, 8>(), near);
        default: return f(type, std::integral_constant<int, 16>(), near);
        }
    };
    auto with_pairs = [&](auto type) {
        if (pairs == MMEE_PAIRS_NEIGHBOURS) with_lanes(type, std::true_type());
        else with_lanes(type, std::false_type());
    };
    if (dtype == MMEE_F16) with_pairs(F16());
    else with_pairs(BF16());
}

// Blocks of one wave while there are few, so that they spread over the card.
struct Grid {
    uint64_t blocks;
    uint32_t threads;
    explicit Grid(uint64_t waves) : blocks(waves <= 1024 ? waves : (waves + 3) / 4), threads(waves <= 1024 ? 64 : 256) {}
};

}  // namespace
}  // namespace mmee

using namespace mmee;

extern "C" {

int mmee_qk_rotate_workspace(const mmee_qk_rotate *x, uint64_t *bytes)
{
    if (!bytes) return MMEE_EINVAL;
    RotateArgs r = {};
    const int rc = plan_rotate(x, false, r);
    if (rc) return rc;
    *bytes = parts_bytes(r);
    return MMEE_OK;
}

int mmee_qk_rotate_forward(const mmee_qk_rotate *x)
{
    RotateArgs r = {};
    const int rc = plan_rotate(x, true, r);
    if (rc) return rc;
    if (!r.tokens) return MMEE_OK;
    const Grid grid((uint64_t)r.tokens * r.shares);
    Launching l;
    if (l.rc) return l.rc;
    dispatch(x->dtype, x->pairs, r.head_dim, [&](auto type, auto lanes, auto near) { l.run(k_rotate<decltype(type), lanes.value, near.value, false>, grid.blocks, grid.threads, r); });
    return l.result("rotation, forward");
}

int mmee_qk_rotate_backward(const mmee_qk_rotate *x, const mmee_qk_rotate_grads *g)
{
    RotateArgs r = {};
    const int rc = plan_rotate(x, true, r);
    if (rc) return rc;
    if (!g || (r.tokens && (!g->dq_out || !g->dk_out || !g->dq || !g->dk)) || (r.q_weight && (!g->dq_weight || !g->dk_weight))) return MMEE_EINVAL;
    if (misaligned({g->dq_out, g->dk_out, g->dq, g->dk, g->dq_weight, g->dk_weight}, 16)) return MMEE_EINVAL;
    if (!take(g->dq_out_stride, r.tokens, r.heads, false, r.dqos) || !take(g->dk_out_stride, r.tokens, r.kv_heads, false, r.dkos) || !take(g->dq_stride, r.tokens, r.heads, true, r.dqs) ||
        !take(g->dk_stride, r.tokens, r.kv_heads, true, r.dks))
        return MMEE_EINVAL;
    if (moved(g->dq_out, r.dqos, g->dq, r.dqs) || moved(g->dk_out, r.dkos, g->dk, r.dks)) return MMEE_EINVAL;
    const uint64_t need = parts_bytes(r);
    if (need && (!x->workspace || x->workspace_bytes < need)) return MMEE_EWORKSPACE;
    r.dq_out = (const uint16_t *)g->dq_out;
    r.dk_out = (const uint16_t *)g->dk_out;
    r.dq = (uint16_t *)g->dq;
    r.dk = (uint16_t *)g->dk;
    r.dq_weight = (uint16_t *)g->dq_weight;
    r.dk_weight = (uint16_t *)g->dk_weight;
    r.parts = (float *)x->workspace;
    if (!r.tokens && !r.q_weight) return MMEE_OK;
    Launching l;
    if (l.rc) return l.rc;
    dispatch(x->dtype, x->pairs, r.head_dim, [&](auto type, auto lanes, auto near) {
        if (r.tokens) l.run(k_rotate_back<decltype(type), lanes.value, near.value>, r.blocks, 256, r);
        if (r.q_weight) l.run(k_rotate_weights<decltype(type)>, (2 * r.head_dim + 31) / 32, 1024, r);
    });
    return l.result("rotation, backward");
}

int mmee_cache_append_forward(const mmee_cache_append *x)
{
    if (!x || x->reserved || !x->seqs || !x->kv_heads || !x->heads != !x->q) return MMEE_EINVAL;
    RotateArgs r = {};
    const int rc = common(x, r);
    if (rc) return rc;
    if (!x->page_tokens || (x->page_tokens & (x->page_tokens - 1)) || x->page_tokens > 1u << 16 || x->n_pages > 0x7fffffff || x->table_stride < 0) return MMEE_EINVAL;
    if (x->seqs > MOST_TOKENS || (!x->starts && x->tokens % x->seqs)) return MMEE_EINVAL;
    if (r.heads ? !x->q_weight != !x->k_weight : x->q_weight != nullptr) return MMEE_EINVAL;
    if (x->rot_dim && !x->positions && (x->axes > 1 || x->axis_of)) return MMEE_EINVAL;
    if (!take(x->q_stride, r.tokens, r.heads, false, r.qs) || !take(x->k_stride, r.tokens, r.kv_heads, false, r.ks) || !take(x->v_stride, r.tokens, r.kv_heads, false, r.vs) ||
        !take(x->q_out_stride, r.tokens, r.heads, r.heads != 0, r.qos) || !take(x->k_pages_stride + 1, x->page_tokens, r.kv_heads, true, r.kos) ||
        !take(x->v_pages_stride + 1, x->page_tokens, r.kv_heads, true, r.vos) || !take(x->k_pages_stride[0], x->n_pages, true, r.k_page) ||
        !take(x->v_pages_stride[0], x->n_pages, true, r.v_page))
        return MMEE_EINVAL;
    if (moved(x->q, r.qs, x->q_out, r.qos)) return MMEE_EINVAL;
    if (r.tokens) {
        if (!x->k || !x->v || !x->cache_lens || (r.heads && !x->q_out) || (x->n_pages && (!x->k_pages || !x->v_pages)) || (x->pages_per_seq && !x->page_table)) return MMEE_EINVAL;
        if (misaligned({x->v, x->k_pages, x->v_pages}, 16) || misaligned({x->starts, x->counts, x->cache_lens, x->page_table}, 4)) return MMEE_EINVAL;
    }
    r.v = (const uint16_t *)x->v;
    r.q_out = (uint16_t *)x->q_out;
    r.k_out = (uint16_t *)x->k_pages;
    r.v_out = (uint16_t *)x->v_pages;
    if (!r.heads) r.q_weight = r.k_weight;      // (never a query's)
    r.starts = x->starts;
    r.counts = x->counts;
    r.cache_lens = x->cache_lens;
    r.page_table = x->page_table;
    r.table_stride = x->seqs > 1 ? x->table_stride : 0;
    r.seqs = x->seqs;
    r.per_seq = std::max(1u, x->tokens / x->seqs);
    while ((1u << r.page_shift) < x->page_tokens) ++r.page_shift;
    r.pages_per_seq = x->pages_per_seq;
    r.n_pages = x->n_pages;
    if (!r.tokens) return MMEE_OK;
    r.shares = shares(r.tokens, r.heads + 2 * r.kv_heads, lanes_of(r.head_dim));
    const Grid grid((uint64_t)r.tokens * r.shares);
    Launching l;
    if (l.rc) return l.rc;
    dispatch(x->dtype, x->pairs, r.head_dim, [&](auto type, auto lanes, auto near) { l.run(k_rotate<decltype(type), lanes.value, near.value, true>, grid.blocks, grid.threads, r); });
    return l.result("appending to the cache");
}

}  // extern "C"
