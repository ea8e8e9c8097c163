// C entry points of the dense layers in bfloat16 or float32 and of the clipping of gradients: validation, workspace layout, order of the launches.
#include "st_clip.hpp"
#include "st_linear.hpp"
#include "st_overlap.hpp"

#include <math.h>
#include <algorithm>

namespace st {
namespace {

// A launch holds fewer than 2^32 threads and 2^23 tiles.
constexpr int64_t MAX_TOKENS = (1 << 24) - 1, MAX_CHANNELS = ST_LINEAR_MAX_CHANNELS, MAX_VALUES = (int64_t)1 << 33, MAX_STRIDE = (int64_t)1 << 40;

struct Carve {      // 256-byte aligned pieces of a workspace
    char* base; size_t used = 0;
    void* take(size_t bytes) { void* p = base + used; used += (bytes + 255) / 256 * 256; return p; }
};
bool dtype_ok(int32_t d) { return d == ST_F32 || d == ST_BF16; }
int elem(int32_t d) { return d == ST_BF16 ? 2 : 4; }
bool is_aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
bool tiles_ok(int64_t a, int64_t b) { return ceil_div(a, 64) * ceil_div(b, 64) < (1 << 23); }
bool sizes_ok(int64_t m, int64_t n, int64_t k)
{
    return m >= 0 && m <= MAX_TOKENS && n >= 1 && n <= MAX_CHANNELS && k >= 1 && k <= MAX_CHANNELS && tiles_ok(m, n) && tiles_ok(m, k) && tiles_ok(n, k);
}

// Whether the matrix can be read, and whether its rows lie along memory (*along).
int check(const st_matrix* x, int64_t rows, int64_t cols, int* along)
{
    if (!x) return ST_ERR_NULL;
    if (x->rows != rows || x->cols != cols) return ST_ERR_SHAPE;
    if (!dtype_ok(x->dtype)) return ST_ERR_ARG;
    if (rows > 0 && !x->data) return ST_ERR_NULL;
    if (!is_aligned(x->data, elem(x->dtype))) return ST_ERR_ARG;
    if (x->row_stride < 0 || x->col_stride < 0 || x->row_stride > MAX_STRIDE || x->col_stride > MAX_STRIDE) return ST_ERR_SHAPE;
    if (x->col_stride == 1 || cols == 1) *along = 1;
    else if (x->row_stride == 1 || rows <= 1) *along = 0;
    else return ST_ERR_SHAPE;
    return ST_OK;
}

// What a call touches: a result row by row, a matrix that lies either way (checked), a vector.  No memory reaches FARTHEST from one run to the next.
constexpr int64_t FARTHEST = (int64_t)1 << 39;
Runs runs_of(const void* p, int32_t dtype, int64_t count, int64_t values, int64_t pitch)
{
    return Runs{(uint64_t)p, count, values * elem(dtype), std::min(pitch, FARTHEST / elem(dtype)) * elem(dtype)};
}
Runs runs_of(const st_matrix& x, int along)
{
    return runs_of(x.data, x.dtype, along ? x.rows : x.cols, along ? x.cols : x.rows, along ? x.row_stride : x.col_stride);
}
Runs runs_of(const float* p, int64_t n) { return Runs{(uint64_t)p, 1, n * 4, 0}; }
// Whether one of the `written` overlaps another or one of the `read` (places at address 0 are not there).
struct Touched {
    Runs written[3], read[5];
    int n_written = 0, n_read = 0;
    void writes(const Runs& r) { if (r.at) written[n_written++] = r; }
    void reads(const Runs& r) { if (r.at) read[n_read++] = r; }
    bool overlap() const
    {
        for (int i = 0; i < n_written; ++i) {
            for (int j = 0; j < i; ++j) if (st::overlap(written[i], written[j])) return true;
            for (int j = 0; j < n_read; ++j) if (st::overlap(written[i], read[j])) return true;
        }
        return false;
    }
};

// An operand whose rows are x's rows (by_rows) or its columns: as it lies, or where the products cannot read it so, a copy that `packs`
// makes (with room in `w`).  The copy lies as x does, unless only the other order keeps a tile's offsets small.
struct Packs { PackTask t[PACK_TASKS]; int n = 0; };
struct Lie { int64_t outer, inner, pitch; int k_along; bool direct; };      // k_along: the operand's rows lie along memory
Lie lie_of(const st_matrix& x, int along, bool by_rows)
{
    Lie l{along ? x.rows : x.cols, along ? x.cols : x.rows, along ? x.row_stride : x.col_stride, along == (by_rows ? 1 : 0), false};
    if (l.outer == 1) l.pitch = round_up(l.inner, 16 / elem(x.dtype));      // (whatever the caller has there)
    l.direct = operand_direct(x.data, l.pitch, l.k_along, l.inner, elem(x.dtype));
    return l;
}
int64_t copied_bytes(const st_matrix& x, int along, bool by_rows)
{
    return lie_of(x, along, by_rows).direct ? 0 : x.rows * x.cols * elem(x.dtype);
}
Operand operand_of(const st_matrix& x, int along, bool by_rows, bool small, int* loose, Carve& w, Packs* packs)
{
    const int es = elem(x.dtype);
    const Lie l = lie_of(x, along, by_rows);
    const int64_t outer = l.outer, inner = l.inner, pitch = l.pitch;
    const int k_along = l.k_along;
    if (l.direct) return Operand{x.data, pitch, k_along, round_up(inner, 16 / es)};      // (whole aligned chunks are there)
    if (small && inner >= 16 / es) { *loose = 1; return Operand{x.data, pitch, k_along, inner}; }
    const bool turn = !operand_direct(nullptr, round_up(inner, 8), k_along, round_up(inner, 8), es);
    const int64_t to_pitch = round_up(turn ? outer : inner, 8);
    void* to = w.take((size_t)(turn ? inner : outer) * to_pitch * es);
    packs->t[packs->n++] = PackTask{x.data, outer, inner, pitch, to, to_pitch, turn};
    return Operand{to, to_pitch, turn ? !k_along : k_along, to_pitch};
}
size_t slab_bytes(const Extent* e, const LinearForm& f, int which)
{
    return f.splits[which] > 1 ? (size_t)f.splits[which] * e[which].m * e[which].n * 4 : 0;
}
// Whether a launch holds the products' blocks (and those of the columns' sums).
bool fits(const Extent* e, int count, const LinearForm& f)
{
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) blocks += ceil_div(e[i].m, f.tile) * ceil_div(e[i].n, f.tile) * f.splits[i];
    return blocks < (1 << 23) - 32768 - 1;
}

// The forward pass, planned: `ws` null for its size alone; bytes 0: more than a launch holds.
struct LinearPlan { LinearProduct p; LinearForm form; Packs packs; bool few; size_t bytes; };
LinearPlan plan_linear(const st_matrix& x, int x_along, const st_matrix& w, int w_along, char* ws)
{
    LinearPlan l{};
    LinearProduct& p = l.p;
    p.m = x.rows; p.n = w.rows; p.k = x.cols;
    const int is_bf16 = x.dtype == ST_BF16;
    Carve c{ws};
    l.few = w_along && linear_few(p.m, p.n, p.k, is_bf16, is_aligned(w.data, 16) && (w.row_stride * elem(w.dtype) % 16 == 0 || p.n == 1));
    const Extent e{p.m, p.n, p.k};
    if (l.few) {
        p.a = Operand{x.data, x_along ? x.row_stride : x.col_stride, x_along, x_along ? p.k : p.m};
        p.b = Operand{w.data, w.row_stride, 1, p.k};
    } else {
        l.form = linear_form(&e, 1, is_bf16, copied_bytes(x, x_along, true) + copied_bytes(w, w_along, true), false);
        const bool small = l.form.tile == SMALL_TILE;
        p.a = operand_of(x, x_along, true, small, &p.loose, c, &l.packs);
        p.b = operand_of(w, w_along, true, small, &p.loose, c, &l.packs);
        p.slabs = (float*)c.take(slab_bytes(&e, l.form, 0));
    }
    l.bytes = l.few || fits(&e, 1, l.form) ? c.used + 256 : 0;
    return l;
}

// How many bfloat16 terms of dz a product beside bfloat16 operands takes, each a contraction of its own: two (2^-16 off at most) where one would
// show, that is beside a float32 dy, and in a float32 result of any dz that one term does not hold.  A bfloat16 result of a bfloat16 dy has one (2^-8):
// what that adds is as large as the rounding that dy has had and the one that the result gets.  8192 tokens 4096 -> 4096, SiLU, the call with its
// dz: both results in bfloat16 502 us and 0.0024 of the 2-norm from 64 bits (exact dz would give 0.0017), dw in float32 723, both 937.
int dz_terms(int dtype, int dy_dtype, int act, int result_dtype)
{
    const bool exact = act == ST_ACT_NONE || act == ST_ACT_RELU;      // dz is dy or zero
    return dtype == ST_BF16 && (dy_dtype == ST_F32 || (!exact && result_dtype == ST_F32)) ? 2 : 1;
}

// The backward pass, planned the same way for the outputs that are asked for, dw and dx of these types.
struct BackwardPlan { LinearProduct p[2]; LinearForm form; int n_products; Packs packs; SlopeTask slope; bool slopes; ColumnSums sums; size_t bytes; };
BackwardPlan plan_backward(const st_matrix* x, int x_along, int dw_dtype, const st_matrix* w, int w_along, int dx_dtype, const st_matrix& dy, int dy_along,
                           int act, int dtype, bool db, char* ws)
{
    BackwardPlan b{};
    Carve c{ws};
    const int64_t m = dy.rows, n = dy.cols;
    const int is_bf16 = dtype == ST_BF16;
    Operand by_tokens{}, by_channels{};      // dz for dx, and for dw
    const bool as_it_is = act == ST_ACT_NONE && dy.dtype == dtype;
    Extent e[2];
    int terms[2], most = 1;
    if (x) { terms[b.n_products] = dz_terms(dtype, dy.dtype, act, dw_dtype); e[b.n_products] = Extent{n, x->cols, m * terms[b.n_products]}; ++b.n_products; }
    if (w) { terms[b.n_products] = dz_terms(dtype, dy.dtype, act, dx_dtype); e[b.n_products] = Extent{m, w->cols, n * terms[b.n_products]}; ++b.n_products; }
    for (int i = 0; i < b.n_products; ++i) most = std::max(most, terms[i]);
    const int64_t copied = (x ? copied_bytes(*x, x_along, false) : 0) + (w ? copied_bytes(*w, w_along, false) : 0)
                           + (as_it_is && w ? copied_bytes(dy, dy_along, true) : as_it_is && x ? copied_bytes(dy, dy_along, false) : 0);
    b.form = b.n_products ? linear_form(e, b.n_products, is_bf16, copied, db || !as_it_is) : LinearForm{SMALL_TILE, {1, 1}};
    const bool small = b.form.tile == SMALL_TILE;
    int loose = 0;
    SlopeTask& s = b.slope;
    s.dy = GradSource{dy.data, dy.dtype == ST_BF16, dy_along ? dy.row_stride : dy.col_stride, dy_along};
    s.act = act; s.m = m; s.n = n; s.to_bf16 = is_bf16;
    b.slopes = db || ((x || w) && !as_it_is);
    if ((x || w) && !as_it_is) {
        s.to_pitch = round_up(n, 8);
        s.second = most == 2 ? m * s.to_pitch : 0;
        s.to = c.take((size_t)m * s.to_pitch * elem(dtype) * most);
        by_tokens = Operand{s.to, s.to_pitch, 1, s.to_pitch};
        by_channels = Operand{s.to, s.to_pitch, 0, s.to_pitch};
    } else {
        if (w) by_tokens = operand_of(dy, dy_along, true, small, &loose, c, &b.packs);
        // the same matrix read the other way round, if it can be (the rows of a copy end in zeros)
        const bool is_copy = b.packs.n > 0;
        const int64_t pitch = by_tokens.pitch;
        if (w && operand_direct(by_tokens.p, pitch, !by_tokens.along, by_tokens.along ? n : is_copy ? round_up(m, 8) : m, elem(dtype)))
            by_channels = Operand{by_tokens.p, pitch, !by_tokens.along, by_tokens.inner};
        else if (x) by_channels = operand_of(dy, dy_along, false, small, &loose, c, &b.packs);
    }
    if (db) {
        s.parts = (float*)c.take((size_t)linear_slope_parts(m, n) * n * 4);
        b.sums = ColumnSums{s.parts, linear_slope_parts(m, n), n, nullptr, 0};
    }
    int at = 0;
    if (x) {
        LinearProduct& p = b.p[at++];
        p.a = by_channels;
        p.b = operand_of(*x, x_along, false, small, &loose, c, &b.packs);
    }
    if (w) {
        LinearProduct& p = b.p[at++];
        p.a = by_tokens;
        p.b = operand_of(*w, w_along, false, small, &loose, c, &b.packs);
    }
    for (int i = 0; i < b.n_products; ++i) { LinearProduct& p = b.p[i]; p.m = e[i].m; p.n = e[i].n; p.k = e[i].k / terms[i]; p.a_second = terms[i] == 2 ? s.second : 0; p.loose = loose; }
    for (int i = 0; i < b.n_products; ++i) b.p[i].slabs = (float*)c.take(slab_bytes(e, b.form, i));
    b.bytes = fits(e, b.n_products, b.form) ? c.used + 256 : 0;
    return b;
}

}  // namespace
}  // namespace st

using namespace st;

extern "C" {

static int check_linear(const st_matrix* x, const st_matrix* w, int* x_along, int* w_along)
{
    if (!x || !w) return ST_ERR_NULL;
    if (!sizes_ok(x->rows, w->rows, x->cols)) return ST_ERR_SHAPE;
    if (const int v = check(x, x->rows, x->cols, x_along)) return v;
    if (const int v = check(w, w->rows, x->cols, w_along)) return v;
    return x->dtype == w->dtype ? ST_OK : ST_ERR_ARG;
}

size_t st_linear_workspace(const st_matrix* x, const st_matrix* w)
{
    int x_along = 1, w_along = 1;
    if (check_linear(x, w, &x_along, &w_along) != ST_OK) return 0;
    return x->rows ? plan_linear(*x, x_along, *w, w_along, nullptr).bytes : 256;
}

int st_linear(const st_matrix* x, const st_matrix* w, const st_linear_opts* opts, void* y, int32_t y_dtype, int64_t y_pitch,
              void* workspace, size_t workspace_bytes, void* stream)
{
    int x_along = 1, w_along = 1;
    if (const int v = check_linear(x, w, &x_along, &w_along)) return v;
    const st_linear_opts none{}, &o = opts ? *opts : none;
    const int64_t n = w->rows;
    if (y_pitch < n || (o.residual && o.residual_pitch < n) || (o.pre && o.pre_pitch < n)) return ST_ERR_SHAPE;
    if (!dtype_ok(y_dtype) || o.activation < ST_ACT_NONE || o.activation > ST_ACT_SILU || (o.residual && !dtype_ok(o.residual_dtype))
        || (o.pre && !dtype_ok(o.pre_dtype)))
        return ST_ERR_ARG;
    if (x->rows == 0) return ST_OK;
    if (!y) return ST_ERR_NULL;
    if (!is_aligned(y, elem(y_dtype)) || !is_aligned(o.bias, 4) || (o.residual && !is_aligned(o.residual, elem(o.residual_dtype)))
        || (o.pre && !is_aligned(o.pre, elem(o.pre_dtype))))
        return ST_ERR_ARG;
    if (o.residual == y && (o.residual_dtype != y_dtype || o.residual_pitch != y_pitch)) return ST_ERR_ARG;
    LinearPlan l = plan_linear(*x, x_along, *w, w_along, (char*)workspace);
    if (!l.bytes) return ST_ERR_SHAPE;
    if (l.bytes > 256 && (!workspace || !is_aligned(workspace, 256) || workspace_bytes < l.bytes)) return ST_ERR_WORKSPACE;
    const int64_t m = x->rows;
    Touched t;
    t.writes(runs_of(y, y_dtype, m, n, y_pitch));
    if (o.pre) t.writes(runs_of(o.pre, o.pre_dtype, m, n, o.pre_pitch));
    t.reads(runs_of(*x, x_along)); t.reads(runs_of(*w, w_along)); t.reads(runs_of(o.bias, n));
    if (o.residual && o.residual != y) t.reads(runs_of(o.residual, o.residual_dtype, m, n, o.residual_pitch));
    if (t.overlap()) return ST_ERR_ARG;
    LinearProduct& p = l.p;
    p.out = y; p.out_bf16 = y_dtype == ST_BF16; p.out_pitch = y_pitch;
    p.bias = o.bias; p.act = o.activation;
    p.residual = o.residual; p.residual_bf16 = o.residual_dtype == ST_BF16; p.residual_pitch = o.residual_pitch;
    p.pre = o.pre; p.pre_bf16 = o.pre_dtype == ST_BF16; p.pre_pitch = o.pre_pitch;
    const int is_bf16 = x->dtype == ST_BF16;
    Ctx c{(hipStream_t)stream, ST_OK};
    if (l.few) { linear_product_few(c, p, is_bf16); return c.status; }
    linear_prepare(c, nullptr, l.packs.t, l.packs.n, is_bf16);
    linear_products(c, &p, 1, l.form, is_bf16, ColumnSums{});
    return c.status;
}

// x and w: those that the gradients asked for need, or null
static int check_backward(const st_matrix* x, const st_matrix* w, const st_matrix* dy, int32_t act, int* x_along, int* w_along, int* dy_along)
{
    if (!dy) return ST_ERR_NULL;
    const int64_t m = dy->rows, n = dy->cols, k = w ? w->cols : x ? x->cols : 1;
    if (!sizes_ok(m, n, k)) return ST_ERR_SHAPE;
    if (act < ST_ACT_NONE || act > ST_ACT_SILU) return ST_ERR_ARG;
    if (const int v = check(dy, m, n, dy_along)) return v;
    if (x) if (const int v = check(x, m, k, x_along)) return v;
    if (w) if (const int v = check(w, n, k, w_along)) return v;
    if (x && w && x->dtype != w->dtype) return ST_ERR_ARG;
    return ST_OK;
}

size_t st_linear_backward_workspace(const st_matrix* x, const st_matrix* w, const st_matrix* dy, int32_t activation)
{
    int x_along = 1, w_along = 1, dy_along = 1;
    if (check_backward(x, w, dy, activation, &x_along, &w_along, &dy_along) != ST_OK) return 0;
    if (dy->rows == 0) return 256;
    const int dtype = x ? x->dtype : w ? w->dtype : dy->dtype;
    size_t most = 0;      // whichever of the gradients are asked for, in whichever type
    const bool types_count = dz_terms(dtype, dy->dtype, activation, ST_F32) != dz_terms(dtype, dy->dtype, activation, ST_BF16);
    for (int which = 0; which < (types_count ? 32 : 8); ++which) {
        if ((which & 8 && !(which & 1)) || (which & 16 && !(which & 2))) continue;
        const size_t bytes = plan_backward(which & 1 ? x : nullptr, x_along, which & 8 ? ST_F32 : ST_BF16, which & 2 ? w : nullptr, w_along, which & 16 ? ST_F32 : ST_BF16,
                                           *dy, dy_along, activation, dtype, which & 4, nullptr).bytes;
        if (!bytes) return 0;
        most = std::max(most, bytes);
    }
    return most;
}

int st_linear_backward(const st_matrix* x, const st_matrix* w, const st_matrix* dy, const st_matrix* pre, int32_t activation,
                       const st_linear_grads* grads, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!grads) return ST_ERR_NULL;
    const st_linear_grads& o = *grads;
    if ((o.dx && !w) || (o.dw && !x)) return ST_ERR_NULL;
    if (!o.dx) w = nullptr;
    if (!o.dw) x = nullptr;
    int x_along = 1, w_along = 1, dy_along = 1, pre_along = 1;
    if (const int v = check_backward(x, w, dy, activation, &x_along, &w_along, &dy_along)) return v;
    const int64_t m = dy->rows, n = dy->cols, k = w ? w->cols : x ? x->cols : 1;
    if (activation != ST_ACT_NONE) if (const int v = check(pre, m, n, &pre_along)) return v;
    if ((o.dx && o.dx_pitch < k) || (o.dw && o.dw_pitch < k)) return ST_ERR_SHAPE;
    if ((o.dx && !dtype_ok(o.dx_dtype)) || (o.dw && !dtype_ok(o.dw_dtype)) || (o.accumulate != 0 && o.accumulate != 1)) return ST_ERR_ARG;
    if ((o.dx && !is_aligned(o.dx, elem(o.dx_dtype))) || (o.dw && !is_aligned(o.dw, elem(o.dw_dtype))) || !is_aligned(o.db, 4)) return ST_ERR_ARG;
    if (!o.dx && !o.dw && !o.db) return ST_OK;
    Ctx c{(hipStream_t)stream, ST_OK};
    if (m == 0) {
        if (o.accumulate) return ST_OK;
        if (o.dw) linear_fill_zero(c, o.dw, o.dw_dtype == ST_BF16, n, k, o.dw_pitch);
        if (o.db) linear_fill_zero(c, o.db, 0, 1, n, n);
        return c.status;
    }
    const int dtype = x ? x->dtype : w ? w->dtype : dy->dtype;
    BackwardPlan b = plan_backward(x, x_along, o.dw_dtype, w, w_along, o.dx_dtype, *dy, dy_along, activation, dtype, o.db != nullptr, (char*)workspace);
    if (!b.bytes) return ST_ERR_SHAPE;
    if (b.bytes > 256 && (!workspace || !is_aligned(workspace, 256) || workspace_bytes < b.bytes)) return ST_ERR_WORKSPACE;
    Touched t;
    if (o.dx) t.writes(runs_of(o.dx, o.dx_dtype, m, k, o.dx_pitch));
    if (o.dw) t.writes(runs_of(o.dw, o.dw_dtype, n, k, o.dw_pitch));
    t.writes(runs_of(o.db, n));
    if (x) t.reads(runs_of(*x, x_along));
    if (w) t.reads(runs_of(*w, w_along));
    t.reads(runs_of(*dy, dy_along));
    if (activation != ST_ACT_NONE) t.reads(runs_of(*pre, pre_along));
    if (t.overlap()) return ST_ERR_ARG;
    if (activation != ST_ACT_NONE) b.slope.pre = GradSource{pre->data, pre->dtype == ST_BF16, pre_along ? pre->row_stride : pre->col_stride, pre_along};
    b.sums.out = o.db; b.sums.accumulate = o.accumulate;
    int at = 0;
    if (x) {
        LinearProduct& p = b.p[at++];
        p.out = o.dw; p.out_bf16 = o.dw_dtype == ST_BF16; p.out_pitch = o.dw_pitch;
        if (o.accumulate) { p.residual = o.dw; p.residual_bf16 = p.out_bf16; p.residual_pitch = o.dw_pitch; }
    }
    if (w) {
        LinearProduct& p = b.p[at++];
        p.out = o.dx; p.out_bf16 = o.dx_dtype == ST_BF16; p.out_pitch = o.dx_pitch;
    }
    linear_prepare(c, b.slopes ? &b.slope : nullptr, b.packs.t, b.packs.n, dtype == ST_BF16);
    linear_products(c, b.p, b.n_products, b.form, dtype == ST_BF16, b.sums);
    return c.status;
}

static int check_grads(const st_grad_tensor* t, int32_t n)
{
    if (n < 0 || n > ST_GRAD_MAX_TENSORS) return ST_ERR_SHAPE;
    if (n && !t) return ST_ERR_NULL;
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].n < 0 || t[i].n > MAX_VALUES) return ST_ERR_SHAPE;
        all += t[i].n;
        if (all > MAX_VALUES) return ST_ERR_SHAPE;
    }
    return ST_OK;
}

size_t st_grad_clip_workspace(const st_grad_tensor* tensors, int32_t n_tensors)
{
    if (check_grads(tensors, n_tensors) != ST_OK) return 0;
    return 256 + (size_t)clip_parts(tensors, n_tensors) * sizeof(double);      // (room for one more: their sum)
}

int st_grad_clip(const st_grad_tensor* tensors, int32_t n_tensors, double grad_scale, double max_norm, float* grad_norm, void* workspace, void* stream)
{
    if (const int v = check_grads(tensors, n_tensors)) return v;
    if (!((float)grad_scale > 0) || !isfinite((float)grad_scale) || !(max_norm >= 0) || !isfinite((float)max_norm)
        || (max_norm > 0 && !((float)max_norm > 0)) || !is_aligned(grad_norm, 4))
        return ST_ERR_ARG;
    int with = 0, without = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const st_grad_tensor& t = tensors[i];
        if (!dtype_ok(t.grad_dtype) || (t.out && !dtype_ok(t.out_dtype))) return ST_ERR_ARG;
        if (t.n == 0) continue;
        if (!t.grad) return ST_ERR_NULL;
        if (!is_aligned(t.grad, elem(t.grad_dtype)) || (t.out && !is_aligned(t.out, elem(t.out_dtype)))) return ST_ERR_ARG;
        ++(t.out ? with : without);
        if (t.out) {      // in place, or apart
            const uintptr_t g = (uintptr_t)t.grad, o = (uintptr_t)t.out;
            if (g == o ? t.grad_dtype != t.out_dtype : g < o + t.n * elem(t.out_dtype) && o < g + t.n * elem(t.grad_dtype)) return ST_ERR_ARG;
        }
    }
    if (with && without) return ST_ERR_NULL;
    if (!with && !grad_norm) return ST_OK;
    if (!workspace || !is_aligned(workspace, 256)) return ST_ERR_WORKSPACE;
    Ctx c{(hipStream_t)stream, ST_OK};
    grad_clip(c, tensors, n_tensors, ClipRule{grad_scale, max_norm, grad_norm, with > 0}, (double*)workspace);
    return c.status;
}

}  // extern "C"
