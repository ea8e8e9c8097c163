// C entry points of the dense layers and of the optimiser step: validation, workspace layout, order of the launches.
#include "st_dense.hpp"

#include <math.h>
#include <algorithm>

namespace st {
namespace {

// A launch holds fewer than 2^32 threads: rows that take a block each, tiles of 512 threads, tiles of an optimiser step.
constexpr int64_t MAX_DIM = (1 << 24) - 1, MAX_PITCH = 1 << 23, MAX_VALUES = (int64_t)1 << 33;

struct Carve {      // 256-byte aligned pieces of a workspace
    char* base; size_t used = 0;
    void* take(size_t bytes) { void* p = base + used; used += (bytes + 255) / 256 * 256; return p; }
    Quantized operand(int64_t rows, int64_t len)
    {
        Quantized q;
        q.pitch = round_up(len, OPERAND_QUANTUM);
        q.q = (int8_t*)take((size_t)rows * q.pitch);
        q.scale = (float*)take((size_t)rows * 4);
        return q;
    }
};

bool dtype_ok(int32_t d) { return d == ST_F32 || d == ST_BF16; }
size_t elem(int32_t d) { return d == ST_BF16 ? 2 : 4; }
bool is_aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// Whether the matrix can be read, and whether its rows lie along memory (*along).
int check(const st_matrix* x, int64_t rows, int64_t cols, int* along)
{
    if (!x) return ST_ERR_NULL;
    if (x->rows != rows || x->cols != cols) return ST_ERR_SHAPE;
    if (!dtype_ok(x->dtype)) return ST_ERR_ARG;
    if (rows > 0 && !x->data) return ST_ERR_NULL;
    if (!is_aligned(x->data, elem(x->dtype))) return ST_ERR_ARG;
    if (x->row_stride < 0 || x->col_stride < 0) return ST_ERR_SHAPE;
    if (x->col_stride == 1 || cols == 1) *along = 1;
    else if (x->row_stride == 1 || rows <= 1) *along = 0;
    else return ST_ERR_SHAPE;
    return ST_OK;
}
bool size_ok(int64_t v, int64_t least) { return v >= least && v <= MAX_DIM; }

// The rows of x as rows of an operand, or with `transposed` its columns.
QuantSource source(const st_matrix& x, int along, bool transposed, const st_matrix* mask = nullptr)
{
    QuantSource s;
    s.x = x.data; s.bf16 = x.dtype == ST_BF16;
    s.rows = transposed ? x.cols : x.rows; s.len = transposed ? x.rows : x.cols;
    s.pitch = along ? x.row_stride : x.col_stride;
    s.along = transposed ? !along : along;
    s.mask = mask ? mask->data : nullptr; s.mask_bf16 = mask && mask->dtype == ST_BF16;
    s.mask_pitch = mask ? (along ? mask->row_stride : mask->col_stride) : 0;
    return s;
}
// scratch of a source that is transposed on the way
size_t parts_bytes(int64_t rows, int64_t len) { return (size_t)transpose_parts(rows, len) * rows * 4; }
// scratch of product `which` of those that share a launch
size_t slab_bytes(const Extent* e, int count, int which)
{
    const Form f = form_of(e, count);
    return f.splits[which] > 1 ? (size_t)f.splits[which] * e[which].m * e[which].n * 4 : 0;
}

struct LinearSpace { Quantized x; float* parts; int* slabs; size_t bytes; };
LinearSpace linear_space(char* ws, int64_t m, int64_t n, int64_t k)
{
    Carve w{ws};
    LinearSpace s;
    s.x = w.operand(m, k);
    s.parts = (float*)w.take(m ? parts_bytes(m, k) : 0);
    const Extent e{m, n, k};
    s.slabs = (int*)w.take(m ? slab_bytes(&e, 1, 0) : 0);
    s.bytes = w.used + 256;
    return s;
}
struct BackwardSpace { Quantized dz, dzt, wt, xt; float *dz_max, *dzt_max, *dzt_sum, *wt_max, *xt_max; int *slabs_x, *slabs_w; size_t bytes; };
BackwardSpace backward_space(char* ws, int64_t m, int64_t n, int64_t k)
{
    Carve w{ws};
    BackwardSpace s;
    s.dz = w.operand(m, n); s.dzt = w.operand(n, m); s.wt = w.operand(k, n); s.xt = w.operand(k, m);
    s.dz_max = (float*)w.take(m ? parts_bytes(m, n) : 0);
    s.dzt_max = (float*)w.take(m ? parts_bytes(n, m) : 0);
    s.dzt_sum = (float*)w.take(m ? parts_bytes(n, m) : 0);
    s.wt_max = (float*)w.take(parts_bytes(k, n));
    s.xt_max = (float*)w.take(m ? parts_bytes(k, m) : 0);
    const Extent e[2] = {{n, k, m}, {m, k, n}};       // dw, dx: either may come alone
    s.slabs_w = (int*)w.take(m ? std::max(slab_bytes(e, 2, 0), slab_bytes(e, 1, 0)) : 0);
    s.slabs_x = (int*)w.take(m ? std::max(slab_bytes(e, 2, 1), slab_bytes(e + 1, 1, 0)) : 0);
    s.bytes = w.used + 256;
    return s;
}
bool tiles_ok(int64_t a, int64_t b) { return ceil_div(a, 64) * ceil_div(b, 64) < (1 << 23); }
bool products_ok(const Extent* e, int count)
{
    const Form f = form_of(e, count);
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) blocks += ceil_div(e[i].m, f.tile) * ceil_div(e[i].n, f.tile) * f.splits[i];
    return blocks < (1 << 23);
}

}  // namespace
}  // namespace st

using namespace st;

extern "C" {

size_t st_int8_quantize_workspace(int64_t rows, int64_t cols)
{
    if (!size_ok(rows, 0) || !size_ok(cols, 1) || !tiles_ok(rows, cols)) return 0;
    return rows ? round_up(parts_bytes(rows, cols), 256) + 256 : 256;
}

int st_int8_quantize(const st_matrix* x, int8_t* q, int64_t q_pitch, float* scale, void* workspace, void* stream)
{
    if (!x) return ST_ERR_NULL;
    if (!size_ok(x->rows, 0) || !size_ok(x->cols, 1) || !tiles_ok(x->rows, x->cols)) return ST_ERR_SHAPE;
    int along = 1;
    if (const int v = check(x, x->rows, x->cols, &along)) return v;
    if (q_pitch < x->cols || q_pitch % 16 || q_pitch > MAX_PITCH) return ST_ERR_SHAPE;
    if (x->rows == 0) return ST_OK;
    if (!q || !scale) return ST_ERR_NULL;
    if (!is_aligned(q, 16) || !is_aligned(scale, 4)) return ST_ERR_ARG;
    if (!along && (!workspace || !is_aligned(workspace, 256))) return ST_ERR_WORKSPACE;
    Ctx c{(hipStream_t)stream, ST_OK};
    const QuantTask task{source(*x, along, false), Quantized{q, q_pitch, scale}, (float*)workspace, nullptr, nullptr};
    quantize(c, &task, 1);
    return c.status;
}

size_t st_int8_linear_workspace(int64_t m, int64_t n, int64_t k)
{
    if (!size_ok(m, 0) || !size_ok(n, 1) || !size_ok(k, 1) || k > ST_INT8_MAX_SUM || !tiles_ok(m, n) || !tiles_ok(m, k)) return 0;
    return linear_space(nullptr, m, n, k).bytes;
}

int st_int8_linear(const st_matrix* x, const int8_t* wq, int64_t w_pitch, const float* w_scale, int64_t n, const float* bias,
                   int32_t relu, void* y, int32_t y_dtype, int64_t y_pitch, void* workspace, void* stream)
{
    if (!x) return ST_ERR_NULL;
    const int64_t m = x->rows, k = x->cols;
    if (!st_int8_linear_workspace(m, n, k)) return ST_ERR_SHAPE;
    int along = 1;
    if (const int v = check(x, m, k, &along)) return v;
    if (w_pitch < k || w_pitch % 16 || w_pitch > MAX_PITCH || y_pitch < n) return ST_ERR_SHAPE;
    if (!dtype_ok(y_dtype) || (relu != 0 && relu != 1)) return ST_ERR_ARG;
    if (m == 0) return ST_OK;
    if (!wq || !w_scale || !y) return ST_ERR_NULL;
    if (!is_aligned(wq, 16) || !is_aligned(w_scale, 4) || !is_aligned(bias, 4) || !is_aligned(y, elem(y_dtype))) return ST_ERR_ARG;
    if (!workspace || !is_aligned(workspace, 256)) return ST_ERR_WORKSPACE;
    const LinearSpace s = linear_space((char*)workspace, m, n, k);
    Ctx c{(hipStream_t)stream, ST_OK};
    const QuantSource tokens = source(*x, along, false);
    const Product p{s.x.q, s.x.pitch, s.x.scale, wq, w_pitch, w_scale, m, n, k, y, y_dtype == ST_BF16, y_pitch, bias, relu, s.slabs};
    if (few_fused(m, n, k, tokens.bf16)) { product_few(c, p, &tokens); return c.status; }
    if (along && narrow_layer(m, n, k)) { product_narrow(c, p, tokens); return c.status; }
    const QuantTask task{tokens, s.x, s.parts, nullptr, nullptr};
    quantize(c, &task, 1);
    if (few_tokens(m, n, k)) product_few(c, p, nullptr); else products(c, &p, 1);
    return c.status;
}

size_t st_int8_linear_backward_workspace(int64_t m, int64_t n, int64_t k)
{
    if (!size_ok(m, 0) || !size_ok(n, 1) || !size_ok(k, 1) || n > MAX_PITCH || k > MAX_PITCH || !tiles_ok(m, n) || !tiles_ok(m, k)
        || !tiles_ok(n, k))
        return 0;
    const Extent e[2] = {{n, k, std::max<int64_t>(m, 1)}, {std::max<int64_t>(m, 1), k, n}};
    if (!products_ok(e, 2) || !products_ok(e, 1) || !products_ok(e + 1, 1)) return 0;
    return backward_space(nullptr, m, n, k).bytes;
}

int st_int8_linear_backward(const st_matrix* x, const st_matrix* w, const st_matrix* dy, const st_matrix* y, void* dx,
                            int32_t dx_dtype, int64_t dx_pitch, float* dw, int64_t dw_pitch, float* db, void* workspace,
                            void* stream)
{
    if (!dy || (dx && !w) || (dw && !x)) return ST_ERR_NULL;
    const int64_t m = dy->rows, n = dy->cols, k = dx ? w->cols : dw ? x->cols : 1;
    if (!st_int8_linear_backward_workspace(m, n, k)) return ST_ERR_SHAPE;
    if (dx && n > ST_INT8_MAX_SUM) return ST_ERR_SHAPE;
    if (dw && m > MAX_PITCH) return ST_ERR_SHAPE;
    int dy_along = 1, y_along = 1, x_along = 1, w_along = 1;
    if (const int v = check(dy, m, n, &dy_along)) return v;
    if (dx) if (const int v = check(w, n, k, &w_along)) return v;
    if (dw) if (const int v = check(x, m, k, &x_along)) return v;
    if (y) {
        if (const int v = check(y, m, n, &y_along)) return v;
        if (y_along != dy_along && m > 1 && n > 1) return ST_ERR_SHAPE;
        // One token: both are read across memory, each with its own step, unless both lie along it.  (With one channel check() has set both.)
        if (m == 1 && !y_along) dy_along = 0;
    }
    if (dx && !dtype_ok(dx_dtype)) return ST_ERR_ARG;
    if ((dx && dx_pitch < k) || (dw && dw_pitch < k)) return ST_ERR_SHAPE;
    if ((dx && !is_aligned(dx, elem(dx_dtype))) || !is_aligned(dw, 4) || !is_aligned(db, 4)) return ST_ERR_ARG;
    if (!workspace || !is_aligned(workspace, 256)) return ST_ERR_WORKSPACE;
    Ctx c{(hipStream_t)stream, ST_OK};
    if (m == 0) {
        if (dw) fill_zero(c, dw, n, k, dw_pitch);
        if (db) fill_zero(c, db, 1, n, n);
        return c.status;
    }
    const BackwardSpace s = backward_space((char*)workspace, m, n, k);
    QuantTask task[4];
    int n_tasks = 0;
    // both readings of dz one after the other, the weights last: 8192 tokens 4096 -> 4096 351 us a call, weights second 357, dz^T last 361
    if (dx) task[n_tasks++] = QuantTask{source(*dy, dy_along, false, y), s.dz, s.dz_max, nullptr, nullptr};
    if (dw || db) task[n_tasks++] = QuantTask{source(*dy, dy_along, true, y), dw ? s.dzt : Quantized{nullptr, 0, nullptr}, s.dzt_max, s.dzt_sum, db};
    if (dw) task[n_tasks++] = QuantTask{source(*x, x_along, true), s.xt, s.xt_max, nullptr, nullptr};
    if (dx) task[n_tasks++] = QuantTask{source(*w, w_along, true), s.wt, s.wt_max, nullptr, nullptr};
    quantize(c, task, n_tasks);
    Product p[2];
    int n_products = 0;
    if (dw) p[n_products++] = Product{s.dzt.q, s.dzt.pitch, s.dzt.scale, s.xt.q, s.xt.pitch, s.xt.scale, n, k, m, dw, 0, dw_pitch, nullptr, 0, s.slabs_w};
    if (dx) p[n_products++] = Product{s.dz.q, s.dz.pitch, s.dz.scale, s.wt.q, s.wt.pitch, s.wt.scale, m, k, n, dx, dx_dtype == ST_BF16, dx_pitch, nullptr, 0, s.slabs_x};
    products(c, p, n_products);
    return c.status;
}

static int check_tensors(const st_adamw_tensor* t, int32_t n)
{
    if (n < 0 || n > ST_ADAMW_MAX_TENSORS) return ST_ERR_SHAPE;
    if (n && !t) return ST_ERR_NULL;
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].n < 0 || t[i].n > MAX_VALUES) return ST_ERR_SHAPE;
        all += t[i].n;
    }
    return all > MAX_VALUES ? ST_ERR_SHAPE : ST_OK;
}

size_t st_adamw_workspace(const st_adamw_tensor* tensors, int32_t n_tensors)
{
    if (check_tensors(tensors, n_tensors) != ST_OK) return 0;
    return 256 + (size_t)adamw_norm_parts(tensors, n_tensors) * sizeof(double);
}

int st_adamw_step(const st_adamw_tensor* tensors, int32_t n_tensors, const st_adamw_opts* opts, void* workspace, void* stream)
{
    if (!opts) return ST_ERR_NULL;
    if (const int v = check_tensors(tensors, n_tensors)) return v;
    const st_adamw_opts& o = *opts;
    if (!dtype_ok(o.param_dtype) || !dtype_ok(o.grad_dtype) || (o.state_bits != 8 && o.state_bits != 32) || o.t < 1) return ST_ERR_ARG;
    if (!isfinite(o.lr) || !(o.beta1 >= 0 && o.beta1 < 1) || !(o.beta2 >= 0 && o.beta2 < 1) || !(o.eps >= 0) || !isfinite(o.eps)
        || !((float)o.grad_scale > 0) || !isfinite((float)o.grad_scale) || !(o.max_norm >= 0) || !isfinite(o.max_norm)
        || (o.max_norm > 0 && !((float)o.max_norm > 0)) || !is_aligned(o.grad_norm, 4))
        return ST_ERR_ARG;
    const size_t pe = elem(o.param_dtype), ge = elem(o.grad_dtype), se = o.state_bits == 8 ? 1 : 4;
    for (int i = 0; i < n_tensors; ++i) {
        const st_adamw_tensor& t = tensors[i];
        if (!isfinite(t.weight_decay)) return ST_ERR_ARG;
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || (o.state_bits == 8 && (!t.m_scale || !t.v_scale))) return ST_ERR_NULL;
        if (!is_aligned(t.param, pe) || !is_aligned(t.grad, ge) || !is_aligned(t.m, se) || !is_aligned(t.v, se) || !is_aligned(t.copy, 2)
            || (o.state_bits == 8 && (!is_aligned(t.m_scale, 4) || !is_aligned(t.v_scale, 4))))
            return ST_ERR_ARG;
    }
    const bool clip = o.max_norm > 0;
    if ((clip || o.grad_norm) && (!workspace || !is_aligned(workspace, 256))) return ST_ERR_WORKSPACE;
    Ctx c{(hipStream_t)stream, ST_OK};
    const double bc1 = 1.0 - pow(o.beta1, (double)o.t), bc2 = 1.0 - pow(o.beta2, (double)o.t);
    const AdamwConstants k{(float)o.beta1, (float)o.beta2, (float)(1.0 - o.beta1), (float)(1.0 - o.beta2), (float)o.eps,
                           (float)(o.lr / bc1), (float)(1.0 / sqrt(bc2)), (float)o.grad_scale, (float)o.max_norm};
    adamw_step(c, tensors, n_tensors, o, k, clip || o.grad_norm ? (char*)workspace : nullptr);
    return c.status;
}

int st_adamw_state(const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n, float* m_out,
                   float* v_out, void* stream)
{
    if (n < 0 || n > MAX_VALUES) return ST_ERR_SHAPE;
    if (n == 0 || (!m_out && !v_out)) return ST_OK;
    if ((m_out && (!m || !m_scale)) || (v_out && (!v || !v_scale))) return ST_ERR_NULL;
    if (!is_aligned(m_out, 4) || !is_aligned(v_out, 4) || !is_aligned(m_scale, 4) || !is_aligned(v_scale, 4)) return ST_ERR_ARG;
    Ctx c{(hipStream_t)stream, ST_OK};
    adamw_state(c, m, m_scale, v, v_scale, n, m_out, v_out);
    return c.status;
}

}  // extern "C"
