// Host side of the attention of packed prompts: argument checks, the choice of tiles and pieces, launches.
#include <algorithm>
#include <cmath>

#include "prompt.h"

namespace mmee {
namespace {

constexpr uint64_t MOST_ROWS = 1u << 28;        // rows of one key/value head, keys: token_of() and row numbers stay exact
constexpr int64_t MOST_TOKEN_STRIDE = 1 << 24;  // a tile's offsets fit 32 bits

bool misaligned(const void *p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

// Strides of a tensor of `tokens` x `heads` rows: 16-byte aligned rows, nothing negative; an output's rows are rows of their own.
bool take_strides(const int64_t *given, uint64_t tokens, uint64_t heads, bool output, Strides &out)
{
    const uint64_t extent[2] = {tokens, heads};
    int64_t s[2];
    for (int k = 0; k < 2; ++k) {
        s[k] = extent[k] > 1 ? given[k] : 0;
        if (s[k] < 0 || s[k] % 8 || s[k] > (int64_t)1 << 46 || (output && extent[k] > 1 && s[k] == 0)) return false;
    }
    if (s[0] > MOST_TOKEN_STRIDE) return false;
    out = {0, s[0], s[1]};
    return true;
}

uint64_t up256(uint64_t x) { return (x + 255) & ~(uint64_t)255; }

// One of the three kernels: waves of a block, slots of tiles a head, blocks; whether it has a plan, and one with pieces.
struct Launch {
    int waves = 4;
    uint64_t slots = 0, parts = 0, blocks = 0, room = 0, step = 0, least = 0;
    bool planned = false, pieces = false, lean = false;
    // Of the kernels that join pieces: 32 rows or keys each of every tile that may have been cut.
    uint64_t cut_blocks(const PromptArgs &p) const { return parts / 2 * p.a.kv_heads * waves; }
    uint64_t plan_bytes() const { return planned ? up256(4 * (ENTRIES + ENTRY * slots + parts / 2)) : 0; }
    // Results of pieces, so many floats a row or key.
    uint64_t parts_bytes(uint64_t kv_heads, uint64_t floats) const { return up256(4 * parts * kv_heads * 32 * waves * floats); }
};

struct Plan {
    PromptArgs p = {};
    int dp = 0, dtype = 0;
    Launch forward, dq, dkv;
    uint64_t forward_bytes = 0, backward_bytes = 0;
};

// Tiles of 32 rows (or keys) a wave, `lines` of them in all; `across`: keys (or rows) in all, `step` of them a step.  The lengths are not known here: a
// sequence is taken to be as long as the average.
Launch plan_launch(uint64_t lines, uint64_t seqs, uint64_t kv_heads, uint64_t across, uint64_t step, bool causal, uint64_t eight_from, bool lean)
{
    Launch l;
    l.waves = eight_from && across / seqs >= eight_from && lines / seqs >= 256 && ((lines / 256 + seqs / 2) * kv_heads > 128 || across / seqs >= 1024) ? 8 : 4;
    l.slots = lines / (32 * l.waves) + seqs;
    // Short sequences: the variant of which four blocks run on a unit.  40 sequences of 23 to 509, 12 heads of 64: 23 us instead of 27.
    l.lean = lean && l.waves == 4 && across / seqs <= 256;
    l.room = l.lean ? 1024 : 2048 / l.waves;
    l.step = step;
    l.least = 512 / step;
    const uint64_t tiles = std::max<uint64_t>(1, lines / (32 * l.waves) + seqs / 2), blocks = tiles * kv_heads, steps = across / seqs / step;
    if (seqs <= PLAN_SEQS && l.slots <= PLAN_TILES) {
        // Four times as many tiles as run at once even out the end by themselves.  A plan without pieces pays where tiles of different lengths take more than
        // one round: dQ, dK and dV of 40 sequences of 23 to 509, 12 heads of 64: 61 us with it, 70 without.
        l.pieces = blocks < 4 * l.room && steps >= 2 * l.least;
        l.planned = l.pieces || ((causal || seqs > 1) && blocks > l.room && blocks * steps >= 3 * l.room);
    }
    if (l.pieces) {
        // all pieces but the last of a tile are a unit's share long at least, and a cut tile has two or more
        l.slots += l.room / kv_heads + 1;
        l.parts = 2 * (l.room / kv_heads + 1);
    }
    l.blocks = l.slots * kv_heads;
    return l;
}

int make_plan(const mmee_prompt_attn *x, bool pointers, Plan &plan)
{
    if (!x || x->reserved) return MMEE_EINVAL;
    if (x->dtype != MMEE_F16 && x->dtype != MMEE_BF16) return MMEE_EINVAL;
    if (!x->seqs || !x->heads || !x->kv_heads || x->heads % x->kv_heads || !x->head_dim || x->head_dim % 8 || x->head_dim > 128) return MMEE_EINVAL;
    if (!(x->scale > 0.0f) || !std::isfinite(x->scale)) return MMEE_EINVAL;
    const uint64_t group = x->heads / x->kv_heads, rows = group * x->q_tokens;
    if (rows > MOST_ROWS || group > 4096 || x->kv_tokens > MOST_ROWS || x->heads > 1u << 24 || x->seqs > 1u << 24) return MMEE_EINVAL;
    PromptArgs &p = plan.p;
    AttnArgs &a = p.a;
    if (!take_strides(x->q_stride, x->q_tokens, x->heads, false, a.qs) || !take_strides(x->k_stride, x->kv_tokens, x->kv_heads, false, a.ks) ||
        !take_strides(x->v_stride, x->kv_tokens, x->kv_heads, false, a.vs) || !take_strides(x->o_stride, x->q_tokens, x->heads, true, a.os))
        return MMEE_EINVAL;
    if (pointers) {
        if (!x->q_starts || (!x->kv_starts && x->kv_tokens != x->q_tokens) || (rows && (!x->q || !x->o)) || (x->kv_tokens && (!x->k || !x->v))) return MMEE_EINVAL;
        if (misaligned(x->q) || misaligned(x->k) || misaligned(x->v) || misaligned(x->o) || misaligned(x->workspace) || misaligned(x->lse, 4) || misaligned(x->q_starts, 4) ||
            misaligned(x->kv_starts, 4))
            return MMEE_EINVAL;
    }
    plan.dtype = (int)x->dtype;
    plan.dp = x->head_dim <= 32 ? 32 : x->head_dim <= 64 ? 64 : 128;
    a.batch = 1;
    a.heads = x->heads;
    a.kv_heads = x->kv_heads;
    a.group = (uint32_t)group;
    // r / group = r * ceil(2^shift / group) >> shift for every r < 2^28, as in attention.hip
    a.group_shift = 32;
    while ((uint64_t)1 << (a.group_shift - 32) < group) ++a.group_shift;
    a.group_inverse = (((uint64_t)1 << a.group_shift) + group - 1) / group;
    a.q_len = x->q_tokens;
    a.rows = (uint32_t)rows;
    a.kv_len = x->kv_tokens;
    a.head_dim = x->head_dim;
    a.scale = x->scale;
    a.scale_log2 = x->scale * LOG2E;
    a.q = (const uint16_t *)x->q;
    a.k = (const uint16_t *)x->k;
    a.v = (const uint16_t *)x->v;
    a.o = (uint16_t *)x->o;
    a.lse = x->lse;
    p.q_starts = x->q_starts;
    p.kv_starts = x->kv_starts ? x->kv_starts : x->q_starts;
    p.seqs = x->seqs;
    p.causal = x->causal != 0;
    p.dies = x->kv_heads % 8 == 0;
    // From how many keys (or rows) on average blocks of eight waves, alone on a unit, are worth it: they read each tile half as often as two blocks of four,
    // which cover each other's beginning and end.  Sequences of 256, 512, 1024, 2048, 4096 over themselves, 32768 in all, 16 heads, eight waves against four,
    // microseconds.  Forward, 128 a head: 161, 208, 323, 557, 1027 : 142, 193, 313, 552, 1033; 64 a head: 93, 125, 192, 334, 631 : 74, 110, 183, 328, 628.
    // With the gradients, dQ, 128 a head: 682, 908, 1398, 2424, 4538 : 666, 882, 1384, 2438, 4623; dK and dV, 128 a head: 682, 908, 1398, 2424, 4538 : 678, 928, 1471,
    // 2665, 4972; 64 a head: 395, 543, 849, 1501, 2817 : 381, 535, 856, 1535, 2910.
    const uint64_t forward_from = plan.dp == 128 ? 4096 : 0, dq_from = plan.dp == 128 ? 2048 : 0, dkv_from = plan.dp == 128 ? 512 : plan.dp == 64 ? 1024 : 0;
    plan.forward = plan_launch(rows, x->seqs, x->kv_heads, x->kv_tokens, 64, p.causal, forward_from, plan.dp <= 64);
    plan.dq = plan_launch(rows, x->seqs, x->kv_heads, x->kv_tokens, 64, p.causal, dq_from, false);
    plan.dkv = plan_launch(x->kv_tokens, x->seqs, x->kv_heads, rows, plan.dp == 128 ? 32 : 64, p.causal, dkv_from, false);
    for (const Launch *l : {&plan.forward, &plan.dq, &plan.dkv})
        if (l->blocks * l->waves * 64 > 0xffffffff) return MMEE_EINVAL;         // a launch's threads
    plan.forward_bytes = plan.forward.plan_bytes() + plan.forward.parts_bytes(x->kv_heads, plan.dp + 1);
    plan.backward_bytes = 2 * up256(4ull * x->kv_heads * rows) + plan.dq.plan_bytes() + plan.dkv.plan_bytes() +
                          std::max(plan.dq.parts_bytes(x->kv_heads, plan.dp), plan.dkv.parts_bytes(x->kv_heads, 2 * plan.dp));
    return MMEE_OK;
}

// Calls f(type, padded head size).
template <class F>
void dispatch(const Plan &plan, F f)
{
    auto with_dp = [&](auto type) {
        if (plan.dp == 32) f(type, std::integral_constant<int, 32>());
        else if (plan.dp == 64) f(type, std::integral_constant<int, 64>());
        else f(type, std::integral_constant<int, 128>());
    };
    if (plan.dtype == MMEE_F16) with_dp(F16());
    else with_dp(BF16());
}

// The kernel's arguments: its plan at `at`, if it has one, which moves on behind it; its pieces' results at `parts`.
PromptArgs with(const PromptArgs &p, const Launch &l, char *&at, float *parts)
{
    PromptArgs q = p;
    q.slots = (uint32_t)l.slots;
    q.parts = (uint32_t)l.parts;
    q.plan = l.planned ? (const uint32_t *)at : nullptr;
    q.a.part_o = parts;
    at += l.plan_bytes();
    return q;
}

void make(PlanArgs &x, int &n, const PromptArgs &p, const Launch &l, bool keys)
{
    if (!l.planned) return;
    x.p = p;
    x.of[n++] = {const_cast<uint32_t *>(p.plan), 32u * l.waves, (uint32_t)l.step, p.slots, p.parts, (uint32_t)l.room, l.pieces ? (uint32_t)l.least : 0, keys};
}

// Calls f(8 or 4 waves), 8 where there is such a kernel.
template <bool EIGHT, class F>
void with_waves(int waves, F f)
{
    if constexpr (EIGHT)
        if (waves == 8) return f(std::integral_constant<int, 8>());
    f(std::integral_constant<int, 4>());
}

template <class T, int DP, int W>
void forward_as(const PromptArgs &p, const Launch &at, Launching &l)
{
    bool done = false;
    if constexpr (DP <= 64 && W == 4)
        if (at.lean) {
            l.run(k_prompt_forward<T, DP, W, true>, at.blocks, 64 * W, p);
            done = true;
        }
    if (!done) l.run(k_prompt_forward<T, DP, W, false>, at.blocks, 64 * W, p);
    if (at.pieces) l.run(k_prompt_join<T, DP, W>, at.cut_blocks(p), 8 * DP, p);
}

template <class T, int DP, int W>
void dq_as(const PromptArgs &p, const Launch &at, Launching &l)
{
    l.run(k_prompt_dq<T, DP, W>, at.blocks, 64 * W, p);
    if (at.pieces) l.run(k_prompt_sum<T, DP, W, 64, false>, at.cut_blocks(p), 8 * DP, p);
}

// Whether a step's 32 rows are whole tokens and lie, like the two statistics, within 32 bits of each other.
bool wide(const AttnArgs &a)
{
    const auto spans = [&](const Strides &s) { return (uint64_t)(32 / a.group) * s.token + (uint64_t)a.group * s.head < 1ull << 30; };
    return 32 % a.group == 0 && spans(a.qs) && spans(a.dos) && (uint64_t)a.kv_heads * a.rows < 1u << 28;
}

template <class T, int DP, int W>
void dkv_as(const PromptArgs &p, const Launch &at, Launching &l)
{
    bool done = false;
    if constexpr (DP == 128 && W == 8 && std::is_same_v<T, BF16>)
        if (wide(p.a)) {
            l.run(k_prompt_dkv_wide, at.blocks, 256, p);
            done = true;
        }
    if (!done) l.run(k_prompt_dkv<T, DP, W>, at.blocks, 64 * W, p);
    if (at.pieces) l.run(k_prompt_sum<T, DP, W, DP == 128 ? 32 : 64, true>, at.cut_blocks(p), 8 * DP, p);
}

}  // namespace
}  // namespace mmee

using namespace mmee;

extern "C" {

int mmee_prompt_attn_workspace(const mmee_prompt_attn *x, int backward, uint64_t *bytes)
{
    if (!bytes) return MMEE_EINVAL;
    Plan plan;
    const int rc = make_plan(x, false, plan);
    if (rc) return rc;
    *bytes = std::max(plan.forward_bytes, backward ? plan.backward_bytes : 0);
    return MMEE_OK;
}

int mmee_prompt_attn_forward(const mmee_prompt_attn *x)
{
    Plan plan;
    const int rc = make_plan(x, true, plan);
    if (rc) return rc;
    if (plan.forward_bytes && (!x->workspace || x->workspace_bytes < plan.forward_bytes)) return MMEE_EWORKSPACE;
    if (!plan.p.a.rows) return MMEE_OK;
    char *at = (char *)x->workspace;
    PromptArgs p = with(plan.p, plan.forward, at, (float *)(at + plan.forward.plan_bytes()));
    p.a.part_lse = p.a.part_o + plan.forward.parts * p.a.kv_heads * 32 * plan.forward.waves * plan.dp;
    PlanArgs plans = {};
    int n = 0;
    make(plans, n, p, plan.forward, false);
    Launching l;
    if (l.rc) return l.rc;
    if (n) l.run(k_prompt_plan, n, PLAN_THREADS, plans);
    dispatch(plan, [&](auto type, auto dp) {
        with_waves<(dp.value == 128)>(plan.forward.waves, [&](auto w) { forward_as<decltype(type), dp.value, w.value>(p, plan.forward, l); });
    });
    return l.result("prompt attention, forward");
}

int mmee_prompt_attn_backward(const mmee_prompt_attn *x, const mmee_prompt_attn_grads *g)
{
    Plan plan;
    const int rc = make_plan(x, true, plan);
    if (rc) return rc;
    AttnArgs &a = plan.p.a;
    if (!g || (a.rows && (!x->lse || !g->d_o || !g->dq)) || (a.kv_len && (!g->dk || !g->dv))) return MMEE_EINVAL;
    if (misaligned(g->d_o) || misaligned(g->dq) || misaligned(g->dk) || misaligned(g->dv)) return MMEE_EINVAL;
    if (!take_strides(g->do_stride, a.q_len, a.heads, false, a.dos) || !take_strides(g->dq_stride, a.q_len, a.heads, true, a.dqs) ||
        !take_strides(g->dk_stride, a.kv_len, a.kv_heads, true, a.dks) || !take_strides(g->dv_stride, a.kv_len, a.kv_heads, true, a.dvs))
        return MMEE_EINVAL;
    if (plan.backward_bytes && (!x->workspace || x->workspace_bytes < plan.backward_bytes)) return MMEE_EWORKSPACE;
    if (!a.rows && !a.kv_len) return MMEE_OK;
    a.o_in = (const uint16_t *)x->o;
    a.lse_in = x->lse;
    a.d_o = (const uint16_t *)g->d_o;
    a.dq = (uint16_t *)g->dq;
    a.dk = (uint16_t *)g->dk;
    a.dv = (uint16_t *)g->dv;
    a.delta = (float *)x->workspace;
    plan.p.lse2 = a.delta + up256(4ull * a.kv_heads * a.rows) / 4;
    char *at = (char *)x->workspace + 2 * up256(4ull * a.kv_heads * a.rows);
    float *parts = (float *)(at + plan.dq.plan_bytes() + plan.dkv.plan_bytes());
    const PromptArgs dq = with(plan.p, plan.dq, at, parts), dkv = with(plan.p, plan.dkv, at, parts);
    PlanArgs plans = {};
    int n = 0;
    make(plans, n, dq, plan.dq, false);
    make(plans, n, dkv, plan.dkv, true);
    Launching l;
    if (l.rc) return l.rc;
    if (n) l.run(k_prompt_plan, n, PLAN_THREADS, plans);
    dispatch(plan, [&](auto type, auto dp) {
        if (a.rows) with_waves<(dp.value == 128)>(plan.dq.waves, [&](auto w) { dq_as<decltype(type), dp.value, w.value>(dq, plan.dq, l); });
        if (a.kv_len) with_waves<(dp.value >= 64)>(plan.dkv.waves, [&](auto w) { dkv_as<decltype(type), dp.value, w.value>(dkv, plan.dkv, l); });
    });
    return l.result("prompt attention, backward");
}

}  // extern "C"
