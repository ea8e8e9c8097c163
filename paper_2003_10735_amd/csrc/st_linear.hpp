// Dense layers in bfloat16 or float32 and the clipping of gradients: what their kernels and entry points share.
#pragma once
#include "st_dense.hpp"
#include "st_mfma.hpp"

namespace st {

// ------------------------------------------------------------------ activations
// Phi(-a) for a >= 0 is e(a) q(1 / (1 + 0.31 a)) with e(a) = exp(-a^2 / 2) and q a polynomial: least squares on the relative error over
// a = 0 .. 40, 2e-7 at most in exact arithmetic.  So the lower tail has a relative accuracy, which 1 + erf loses; what limits it far out is the rounding
// of the exponential's argument, here and in the sigmoids below: x steps of 2^-24 of an argument x (to base 2), 2.5 x ln 2 2^-24 of the result at
// most, 7e-6 at a = 10 and 1.2e-5 at 13, where it vanishes.
__device__ __forceinline__ float normal_tail(float a, float* density_shape)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.31f, a, 1.f));
    float q = 0.036023664974412645f;
    q = fmaf(q, t, -0.1425757969074241f);
    q = fmaf(q, t, 0.15717643376193055f);
    q = fmaf(q, t, -0.01733863646625863f);
    q = fmaf(q, t, 0.11174255691275305f);
    q = fmaf(q, t, 0.10712416891165771f);
    q = fmaf(q, t, 0.12420719817577966f);
    q = fmaf(q, t, 0.12363963287446048f);
    q = fmaf(q, t, 7.951515698751551e-07f);
    const float e = __builtin_amdgcn_exp2f(a * a * -0.72134752044448170f);      // log2(e) / 2
    *density_shape = e;
    return e * q;
}
constexpr float LOG2E = 1.4426950408889634f;
// GELU's tanh form is z / (1 + exp(-2 c (z + 0.044715 z^3))) with c = sqrt(2 / pi), since 1 + tanh(u) = 2 / (1 + exp(-2u))
constexpr float TANH_A = -2.f * 0.79788456080286536f * LOG2E, TANH_B = TANH_A * 0.044715f;
__device__ __forceinline__ float sigmoid_of_exp2(float e) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(e)); }

// act(z).  Where z is -infinity the factor is 0 and the result 0, its limit; a NaN stays one.
template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == ST_ACT_RELU) return z < 0.f ? 0.f : z;
    const float low = fmaxf(z, -1e30f);      // (a NaN's factor is a NaN)
    if constexpr (ACT == ST_ACT_GELU) {
        float e;
        const float tail = normal_tail(fabsf(z), &e);
        return low * (z < 0.f ? tail : 1.f - tail);
    }
    if constexpr (ACT == ST_ACT_GELU_TANH) return low * sigmoid_of_exp2(z * fmaf(z * z, TANH_B, TANH_A));
    if constexpr (ACT == ST_ACT_SILU) return low * sigmoid_of_exp2(z * -LOG2E);
    return z;
}
// dy act'(z).  ReLU lets through what lies above zero and nothing else, whatever dy is (a NaN of z lets nothing through).  The other slopes
// have reached 0 or 1 long before |z| = 100, where the factor beside the sigmoid's slope stops growing: infinities give the limit.
template <int ACT> __device__ __forceinline__ float slope_times(float dy, float z)
{
    if constexpr (ACT == ST_ACT_NONE) return dy;
    if constexpr (ACT == ST_ACT_RELU) return z > 0.f ? dy : 0.f;
    const float zc = fminf(fmaxf(z, -100.f), 100.f);
    if constexpr (ACT == ST_ACT_GELU) {
        float e;
        const float tail = normal_tail(fabsf(z), &e);
        return dy * fmaf(zc, e * 0.39894228040143268f, z < 0.f ? tail : 1.f - tail);
    }
    if constexpr (ACT == ST_ACT_GELU_TANH) {
        const float p = sigmoid_of_exp2(z * fmaf(z * z, TANH_B, TANH_A));
        return dy * fmaf(zc * p * (1.f - p), 2.f * 0.79788456080286536f * fmaf(zc * zc, 3.f * 0.044715f, 1.f), p);
    }
    const float p = sigmoid_of_exp2(z * -LOG2E);
    return dy * fmaf(zc * p, 1.f - p, p);
}

// ------------------------------------------------------------------ operands of a product
// Rows of an operand, `pitch` elements apart: along == 1, a row's values (the contraction) lie next to each other; 0: the values of one
// position of the contraction do.  inner: how many values next to each other can be read, 16 bytes of them at least.
struct Operand { const void* p; int64_t pitch; int along; int64_t inner; };
// What the products take of a matrix with `inner` values next to each other: 16-byte aligned, whole 16-byte chunks between two runs, a
// contraction of whole chunks where it lies along memory, and tiles that 32-bit offsets reach.  (Across, a position behind the last one has
// to lie behind the buffer's end: runs do not overlap.)
inline bool operand_direct(const void* p, int64_t pitch, int along, int64_t inner, int es)
{
    const int64_t chunk = 16 / es;
    return (uintptr_t)p % 16 == 0 && pitch % chunk == 0
           && (along ? inner % chunk == 0 && pitch * es < (1 << 23) : pitch >= round_up(inner, chunk) && pitch * es < (1 << 25));
}

// out [m, n] = act(sum_k a[m][k] b[n][k] + bias[n]) + residual[m][n], and beside it the sums with bias alone
struct LinearProduct {
    Operand a, b;                // rows of a: tokens, of b: channels
    int64_t m, n, k;
    void* out; int out_bf16; int64_t out_pitch;
    const float* bias; int act;
    const void* residual; int residual_bf16; int64_t residual_pitch;
    void* pre; int pre_bf16; int64_t pre_pitch;
    float* slabs;                // [splits, m, n] where the contraction is split
    int64_t a_second;            // > 0: a has a second term, that many elements behind the first, whose product with b is added
    int loose;                   // an operand that the products' 16-byte loads do not take as it lies: small tiles load it through registers
};
// Sums of columns that lie as parts: out[i] (+)= sum over the parts of parts[part][i].  Done by the launch of the products.
struct ColumnSums { const float* parts; int n_parts; int64_t n; float* out; int accumulate; };

constexpr int SMALL_TILE = 32;      // small tiles take operands at any address (but rows of less than 16 bytes)
struct LinearForm { int tile; int splits[2]; };
// copied: bytes of operands that small tiles take as they lie and others want copied; prepared: a launch that could copy them is there anyway
LinearForm linear_form(const Extent* e, int count, int is_bf16, int64_t copied, bool prepared);
// up to two products of that form, and sums of columns (n == 0: none), in one launch, and one more where a contraction is split
void linear_products(Ctx& c, const LinearProduct* p, int count, const LinearForm& f, int is_bf16, const ColumnSums& sums);
// few tokens, weights along the contraction: one launch of its own kind, whatever the alignment.  aligned: rows of whole 16-byte chunks
bool linear_few(int64_t m, int64_t n, int64_t k, int is_bf16, bool aligned);
void linear_product_few(Ctx& c, const LinearProduct& p, int is_bf16);

// ------------------------------------------------------------------ operands made for a product
// `outer` runs of `inner` values, `pitch` elements apart, copied to runs that begin at multiples of 16 bytes, zeros up to whole chunks.  With
// `turn` the copy lies the other way round: `inner` runs of `outer` values.
struct PackTask { const void* x; int64_t outer, inner, pitch; void* to; int64_t to_pitch; int turn; };
constexpr int PACK_TASKS = 4;
void linear_fill_zero(Ctx& c, void* p, int is_bf16, int64_t rows, int64_t cols, int64_t pitch);

// dz = dy act'(pre) row by row with zeros up to whole chunks (to null: not stored), and the sums of its columns as parts.  second > 0: what a
// rounding to bfloat16 leaves of it as a second term, that many elements behind the first.
struct GradSource { const void* x; int bf16; int64_t pitch; int along; };
struct SlopeTask {
    GradSource dy, pre;          // pre.x null without activation
    int act; int64_t m, n;
    void* to; int to_bf16; int64_t to_pitch, second;
    float* parts;                // [linear_slope_parts(m, n), n] or null
};
int linear_slope_parts(int64_t m, int64_t n);
// dz (or null) and the copies, in one launch
void linear_prepare(Ctx& c, const SlopeTask* slope, const PackTask* t, int count, int is_bf16);

}  // namespace st
