// Host side of the gated feed-forward block: argument checks, the choice of variant and pieces, launches.
#include <algorithm>
#include <type_traits>

#include "ffn.h"

namespace mmee {
namespace {

constexpr uint32_t MOST_WIDTH = 1u << 22;       // columns and row strides: a tile's offsets fit 32 bits
constexpr uint32_t FEW_TOKENS = 64;

uint64_t up256(uint64_t x) { return (x + 255) & ~(uint64_t)255; }

bool bad_rows(int64_t ld, uint64_t width, uint64_t rows) { return rows > 1 && (ld < (int64_t)width || ld % 8 || ld > (int64_t)MOST_WIDTH); }

bool misaligned(std::initializer_list<const void *> list)
{
    for (const void *p : list)
        if ((uintptr_t)p & 15) return true;
    return false;
}

// A product and how it is run.
struct Job {
    ProductArgs p = {};
    bool big = false;                           // tiles of 256 x 256, else 128 x 128
    bool shared = false;                        // few tokens: through shared memory
    uint32_t columns = 0;                       // few tokens: of a block
    uint32_t blocks = 0;
    uint64_t parts_bytes() const { return p.splits > 1 ? up256(4ull * p.problems * p.splits * p.m * p.n) : 0; }
};

// What a product is estimated to take, in us.  Measured (eight shapes of 128 to 8192 tokens, 768 to 12288 wide, all six products of a
// step, both tiles, one to eight pieces): a step of 64 takes 0.53 us with one tile of 128 x 128 on a compute unit, 1.1 us with two; 1.85 us
// with a tile of 256 x 256 on every one, 1.35 us while half of them have none.  A tile's first loads and its results add 4 us (128) or 7 us (256), 2 and
// 11 us more where results come in two or three tensors.  Pieces are written and read once more in 32 bits.
double estimate(bool big, uint64_t tiles, uint64_t steps, uint64_t splits, uint64_t results, bool many_results)
{
    const uint64_t blocks = tiles * splits, slots = big ? 256 : 512, whole = blocks / slots, rest = blocks % slots;
    const double full = big ? 1.85 : 1.1, half = big ? 1.35 : 0.53, each = (double)((steps + splits - 1) / splits);
    const double last = !rest ? 0.0 : rest <= slots / 2 ? half : full;
    const double ends = (whole + (rest ? 1 : 0)) * (big ? (many_results ? 18.0 : 7.0) : (many_results ? 6.0 : 4.0));
    return each * (whole * full + last) + ends + (splits > 1 ? 3.5 + results * splits * (4.0 / 6e6 + 4.0 / 8e6) : 0.0);
}

// Tiles and pieces of a product: those that are estimated to take least.
bool plan(Job &j, uint32_t m, uint32_t n, uint32_t k, uint32_t segments, uint32_t problems, bool gated, bool may_split)
{
    ProductArgs &p = j.p;
    p.m = m;
    p.n = n;
    p.k = k;
    p.segments = segments;
    p.problems = problems;
    const uint64_t steps = (uint64_t)((k + BK - 1) / BK) * segments;
    const auto tiles = [&](uint32_t side) { return (uint64_t)((m + side - 1) / side) * ((n + side / (gated ? 2 : 1) - 1) / (side / (gated ? 2 : 1))) * problems; };
    double least = 0;
    for (const bool big : {true, false})
        for (uint64_t splits = 1; splits == 1 || (may_split && splits <= 16 && splits * 4 <= steps); ++splits) {
            const double t = estimate(big, tiles(big ? 256 : 128), steps, splits, (uint64_t)m * n * problems, !may_split);
            if (least == 0 || t < least) {
                least = t;
                j.big = big;
                p.splits = (uint32_t)splits;
            }
        }
    const uint32_t tm = j.big ? 256 : 128, tn = tm / (gated ? 2 : 1);
    p.tiles_m = (m + tm - 1) / tm;
    p.tiles_n = (n + tn - 1) / tn;
    const uint64_t blocks = tiles(tm) * p.splits;
    j.blocks = (uint32_t)blocks;
    return blocks <= 0x7fffffff;
}

// Few tokens.  Up to 8 read their operands with the weights; more of them share them (k_tokens_shared: 37 tokens, 4096 -> 12288 -> 4096: 108 -> 75
// us; 16 tokens 79 -> 70), but for gated products too narrow for a block of 32 columns on most compute units, where eight waves on 16 columns are
// sooner done (3072 columns, 37 tokens: 6.6 against 8.8 us).  A block takes 64 columns where that leaves 192 blocks, pieces of the sum counted.
bool plan_tokens(Job &j, uint32_t m, uint32_t n, uint32_t k, bool gated)
{
    ProductArgs &p = j.p;
    p.m = m;
    p.n = n;
    p.k = k;
    p.segments = p.problems = p.splits = 1;
    const uint64_t steps = (k + 31) / 32;
    j.shared = m > 8 && (!gated || n >= 32 * 192);
    uint64_t most = 1;
    if (j.shared) {
        most = gated ? 1 : std::max<uint64_t>(1, std::min<uint64_t>(steps / 16, 16));
        j.columns = n / 64 * most >= 192 ? 64 : 32;
    } else {
        most = gated ? 1 : std::max<uint64_t>(1, std::min<uint64_t>(steps / 32, 16));
        j.columns = n / 32 >= 256 ? 32 : 16;
    }
    const uint64_t blocks = (n + j.columns - 1) / j.columns;
    if (blocks < 192) p.splits = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((j.shared ? 256 : 512) / blocks, most));
    j.blocks = (uint32_t)(blocks * p.splits);
    return true;
}

struct FfnPlan {
    bool tokens = false;                        // few tokens: weights are streamed
    Job hidden, down, d_hidden, dx, dw_gated, dw_down;
    BoundArgs bounds = {};                      // float16, backward
    uint64_t forward_bytes = 0, backward_bytes = 0, d_hidden_bytes = 0, parts_bytes = 0;
    uint64_t bound_blocks() const { return (uint64_t)bounds.row_blocks + bounds.kept_blocks + (uint64_t)bounds.chunks * bounds.strips; }
};

int plan_ffn(const mmee_ffn *x, bool pointers, FfnPlan &f)
{
    if (!x || x->reserved) return MMEE_EINVAL;
    if ((x->dtype != MMEE_F16 && x->dtype != MMEE_BF16) || x->act >= N_ACTS) return MMEE_EINVAL;
    for (const uint32_t width : {x->in_dim, x->hidden_dim, x->out_dim})
        if (!width || width % 8 || width > MOST_WIDTH) return MMEE_EINVAL;
    if (x->rows > 1u << 28) return MMEE_EINVAL;
    if (bad_rows(x->x_stride, x->in_dim, x->rows) || bad_rows(x->gate_stride, x->in_dim, x->hidden_dim) || bad_rows(x->up_stride, x->in_dim, x->hidden_dim) ||
        bad_rows(x->down_stride, x->hidden_dim, x->out_dim) || bad_rows(x->y_stride, x->out_dim, x->rows))
        return MMEE_EINVAL;
    if (x->gate_stride != x->up_stride && x->hidden_dim > 1) return MMEE_EINVAL;
    if (pointers) {
        if (!x->w_gate || !x->w_up || !x->w_down || (x->rows && (!x->x || !x->y || !x->hidden))) return MMEE_EINVAL;
        if (misaligned({x->x, x->w_gate, x->w_up, x->w_down, x->y, x->hidden, x->gate, x->up, x->workspace})) return MMEE_EINVAL;
    }
    const uint32_t M = x->rows, K = x->in_dim, F = x->hidden_dim, J = x->out_dim;
    f.tokens = M <= FEW_TOKENS;
    bool fits = true;
    if (f.tokens) fits = plan_tokens(f.hidden, M, F, K, true) && plan_tokens(f.down, M, J, F, false);
    else fits = plan(f.hidden, M, F, K, 1, 1, true, false) && plan(f.down, M, J, F, 1, 1, false, true);
    fits = fits && plan(f.d_hidden, M, F, J, 1, 1, false, false) && plan(f.dx, M, K, F, 2, 1, false, true) && plan(f.dw_gated, F, K, M, 1, 2, false, true) &&
           plan(f.dw_down, J, F, M, 1, 1, false, true);
    if (!fits) return MMEE_EINVAL;
    f.forward_bytes = f.down.parts_bytes();
    f.d_hidden_bytes = up256(2ull * M * F);
    f.parts_bytes = std::max({f.dx.parts_bytes(), f.dw_gated.parts_bytes(), f.dw_down.parts_bytes()});
    f.backward_bytes = 2 * f.d_hidden_bytes + f.parts_bytes;
    if (x->dtype == MMEE_F16 && M) {
        BoundArgs &b = f.bounds;
        b.rows = M;
        b.hidden = F;
        b.out = J;
        b.row_blocks = (uint32_t)std::min<uint64_t>(512, ((uint64_t)M + 3) / 4);
        b.kept_blocks = (uint32_t)std::min<uint64_t>(1024, ((uint64_t)M * F + 8191) / 8192);
        b.chunks = (J + 63) / 64;
        b.strips = (F + 511) / 512;
        if (f.bound_blocks() > 0x7fffffff) return MMEE_EINVAL;
        f.backward_bytes += up256(4 * (f.bound_blocks() + b.kept_blocks)) + 256;
    }
    return MMEE_OK;
}

template <class T, bool A_ACROSS, bool B_ACROSS, int EPI>
void product(const Job &j, Launching &l)
{
    if (!j.blocks) return;
    if (j.big) l.run(k_product<T, 256, 256, 2, 2, A_ACROSS, B_ACROSS, EPI>, j.blocks, 256, j.p);
    else l.run(k_product<T, 128, 128, 2, 2, A_ACROSS, B_ACROSS, EPI>, j.blocks, 256, j.p);
}

template <class T>
void sum_parts(const Job &j, Launching &l)
{
    if (j.blocks && j.p.splits > 1)
        l.run(k_sum_parts<T>, ((uint64_t)j.p.problems * j.p.m * (j.p.n / 4) + 255) / 256, 256, j.p);
}

template <class T, bool GATED>
void tokens(const Job &j, Launching &l)
{
    auto with = [&](auto mt) {
        constexpr int MT = mt.value;
        if (j.shared && j.columns == 64) l.run(k_tokens_shared<T, MT, 2, 2, GATED>, j.blocks, 512, j.p);
        else if (j.shared) l.run(k_tokens_shared<T, MT, 1, 2, GATED>, j.blocks, 512, j.p);
        else if (GATED && j.columns == 16) l.run(k_tokens<T, GATED ? MT : 1, 1, GATED>, j.blocks, 512, j.p);
        else if (j.columns == 16) l.run(k_tokens<T, 1, 1, GATED>, j.blocks, 512, j.p);
        else l.run(k_tokens<T, 1, 2, GATED>, j.blocks, 512, j.p);          // (up to 8 tokens)
    };
    if (j.p.m <= 16) with(std::integral_constant<int, 1>());
    else if (j.p.m <= 32) with(std::integral_constant<int, 2>());
    else if (j.p.m <= 48) with(std::integral_constant<int, 3>());
    else with(std::integral_constant<int, 4>());
}

template <class T>
void forward_as(const FfnPlan &f, Launching &l)
{
    if (f.tokens) {
        tokens<T, true>(f.hidden, l);
        tokens<T, false>(f.down, l);
    } else {
        product<T, false, false, EPI_GATED>(f.hidden, l);
        product<T, false, false, EPI_STORE>(f.down, l);
    }
    sum_parts<T>(f.down, l);
}

template <class T>
void backward_as(const FfnPlan &f, Launching &l)
{
    if constexpr (NARROW<T>) {
        if (f.bounds.rows) {
            l.run(k_grad_bounds<T>, f.bound_blocks(), 256, f.bounds);
            l.run(k_grad_scale, 1, 1024, f.bounds);
        }
    }
    product<T, false, true, EPI_DGATED>(f.d_hidden, l);
    product<T, false, true, EPI_STORE>(f.dx, l);
    sum_parts<T>(f.dx, l);
    product<T, true, true, EPI_STORE>(f.dw_gated, l);
    sum_parts<T>(f.dw_gated, l);
    product<T, true, true, EPI_STORE>(f.dw_down, l);
    sum_parts<T>(f.dw_down, l);
}

int64_t stride_of(int64_t given, uint64_t rows) { return rows > 1 ? given : 0; }

}  // namespace
}  // namespace mmee

using namespace mmee;

extern "C" {

int mmee_ffn_workspace(const mmee_ffn *x, int backward, uint64_t *bytes)
{
    if (!bytes) return MMEE_EINVAL;
    FfnPlan f;
    const int rc = plan_ffn(x, false, f);
    if (rc) return rc;
    *bytes = backward ? std::max(f.forward_bytes, f.backward_bytes) : f.forward_bytes;
    return MMEE_OK;
}

int mmee_ffn_forward(const mmee_ffn *x)
{
    FfnPlan f;
    const int rc = plan_ffn(x, true, f);
    if (rc) return rc;
    if (f.forward_bytes && (!x->workspace || x->workspace_bytes < f.forward_bytes)) return MMEE_EWORKSPACE;
    if (!x->rows) return MMEE_OK;
    ProductArgs &h = f.hidden.p, &d = f.down.p;
    h.a[0] = (const uint16_t *)x->x;
    h.lda = stride_of(x->x_stride, x->rows);
    h.b[0] = (const uint16_t *)x->w_gate;
    h.b[1] = (const uint16_t *)x->w_up;
    h.ldb = x->gate_stride;
    h.c[0] = (uint16_t *)x->hidden;
    h.ldc = h.ld_hidden = x->hidden_dim;
    h.gate = (uint16_t *)x->gate;
    h.up = (uint16_t *)x->up;
    h.act = (int)x->act;
    d.a[0] = (const uint16_t *)x->hidden;
    d.lda = x->hidden_dim;
    d.b[0] = (const uint16_t *)x->w_down;
    d.ldb = x->down_stride;
    d.c[0] = (uint16_t *)x->y;
    d.ldc = stride_of(x->y_stride, x->rows);
    d.parts = (float *)x->workspace;
    Launching l;
    if (l.rc) return l.rc;
    if (x->dtype == MMEE_F16) forward_as<F16>(f, l);
    else forward_as<BF16>(f, l);
    return l.result("gated feed-forward block, forward");
}

int mmee_ffn_backward(const mmee_ffn *x, const mmee_ffn_grads *g)
{
    FfnPlan f;
    const int rc = plan_ffn(x, true, f);
    if (rc) return rc;
    if (!g || !g->dw_gate || !g->dw_up || !g->dw_down || (x->rows && (!x->gate || !x->up || !g->dy || !g->dx))) return MMEE_EINVAL;
    if (misaligned({g->dy, g->dx, g->dw_gate, g->dw_up, g->dw_down})) return MMEE_EINVAL;
    if (bad_rows(g->dy_stride, x->out_dim, x->rows) || bad_rows(g->dx_stride, x->in_dim, x->rows)) return MMEE_EINVAL;
    if (f.backward_bytes && (!x->workspace || x->workspace_bytes < f.backward_bytes)) return MMEE_EWORKSPACE;
    const int64_t F = x->hidden_dim, K = x->in_dim;
    uint16_t *dg = (uint16_t *)x->workspace, *du = dg + f.d_hidden_bytes / 2;
    float *parts = (float *)(du + f.d_hidden_bytes / 2);
    const int64_t x_stride = stride_of(x->x_stride, x->rows), dy_stride = stride_of(g->dy_stride, x->rows);

    BoundArgs &b = f.bounds;
    if (b.rows) {
        b.dy = (const uint16_t *)g->dy;
        b.ld_dy = dy_stride;
        b.w_down = (const uint16_t *)x->w_down;
        b.ld_down = x->down_stride;
        b.gate = (const uint16_t *)x->gate;
        b.up = (const uint16_t *)x->up;
        b.act = (int)x->act;
        b.scale = parts + f.parts_bytes / 4;
        b.parts = b.scale + 64;
    }

    ProductArgs &h = f.d_hidden.p;
    h.scale = b.scale;
    h.a[0] = (const uint16_t *)g->dy;
    h.lda = dy_stride;
    h.b[0] = (const uint16_t *)x->w_down;
    h.ldb = x->down_stride;
    h.c[0] = dg;
    h.c[1] = du;
    h.ldc = h.ld_hidden = F;
    h.gate_in = (const uint16_t *)x->gate;
    h.up_in = (const uint16_t *)x->up;
    h.act = (int)x->act;

    ProductArgs &dx = f.dx.p;
    dx.scale = b.scale;
    dx.a[0] = dg;
    dx.a[1] = du;
    dx.lda = F;
    dx.b[0] = (const uint16_t *)x->w_gate;
    dx.b[1] = (const uint16_t *)x->w_up;
    dx.ldb = x->gate_stride;
    dx.c[0] = (uint16_t *)g->dx;
    dx.ldc = stride_of(g->dx_stride, x->rows);
    dx.parts = parts;

    ProductArgs &dw = f.dw_gated.p;
    dw.scale = b.scale;
    dw.a[0] = dg;
    dw.a[1] = du;
    dw.lda = F;
    dw.b[0] = (const uint16_t *)x->x;
    dw.ldb = x_stride;
    dw.c[0] = (uint16_t *)g->dw_gate;
    dw.c[1] = (uint16_t *)g->dw_up;
    dw.ldc = K;
    dw.parts = parts;

    ProductArgs &dd = f.dw_down.p;
    dd.a[0] = (const uint16_t *)g->dy;
    dd.lda = dy_stride;
    dd.b[0] = (const uint16_t *)x->hidden;
    dd.ldb = F;
    dd.c[0] = (uint16_t *)g->dw_down;
    dd.ldc = F;
    dd.parts = parts;

    Launching l;
    if (l.rc) return l.rc;
    if (x->dtype == MMEE_F16) backward_as<F16>(f, l);
    else backward_as<BF16>(f, l);
    return l.result("gated feed-forward block, backward");
}

}  // extern "C"
