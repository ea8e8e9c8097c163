// Dense layers in 8-bit integers and the optimiser step over many tensors: what their kernels and entry points share.
#pragma once
#include "st_common.hpp"

namespace st {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_4 __attribute__((aligned(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

inline int64_t round_up(int64_t v, int64_t q) { return (v + q - 1) / q * q; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ quantised operands
// An operand of a product: rows of int8 along the contraction, `pitch` bytes apart, with a scale each.
struct Quantized { int8_t* q; int64_t pitch; float* scale; };

// A matrix to be quantised row by row.  `rows` are the rows of the product's operand, `len` the contraction.
struct QuantSource {
    const void* x; int bf16; int64_t rows, len;
    int64_t pitch;               // elements between two rows (along == 1) or two positions of the contraction (along == 0)
    int along;                   // 1: a row's values lie next to each other; 0: the values of one contraction position do
    const void* mask; int mask_bf16; int64_t mask_pitch;   // keep x where mask > 0; laid out as x; or null
};

constexpr int64_t OPERAND_QUANTUM = 128;         // internal operands: rows of whole stages of the product
// Sources with along == 0 are transposed: the contraction is cut into parts, each of which leaves a largest value (and a sum) per row.
int transpose_parts(int64_t rows, int64_t len);
struct QuantTask {
    QuantSource s;
    Quantized to;                  // q null: only the sums
    float *part_max, *part_sum;    // [parts, rows] where along == 0 (part_sum: where sum is asked for)
    float* sum;                    // [rows]: the plain sums of the rows, or null
};
void quantize(Ctx& c, const QuantTask* tasks, int n);      // up to four

// ------------------------------------------------------------------ products
// out [m, n] = act((sum_k a[m][k] b[n][k]) * a_scale[m] * b_scale[n] + bias[n]).  a's rows hold zeros from k up to a multiple of
// OPERAND_QUANTUM inside their pitch; b's rows are read up to k rounded up to 16.
struct Product {
    const int8_t* a; int64_t a_pitch; const float* a_scale;
    const int8_t* b; int64_t b_pitch; const float* b_scale;
    int64_t m, n, k;
    void* out; int out_bf16; int64_t out_pitch;
    const float* bias; int relu;
    int* slabs;                  // [splits, m, n], see below
};
// Up to two products share a launch: one tile, and for each a number of parts that its contraction is split into.  A split product needs
// splits * m * n ints for the parts' sums.
struct Extent { int64_t m, n, k; };
struct Form { int tile; int splits[2]; };
Form form_of(const Extent* e, int count);
void products(Ctx& c, const Product* p, int count);
// One product of few tokens: a launch of its own kind.  x: the tokens, which it quantises itself; null: p.a holds their codes.
bool few_tokens(int64_t m, int64_t n, int64_t k);
bool few_fused(int64_t m, int64_t n, int64_t k, int is_bf16);
void product_few(Ctx& c, const Product& p, const QuantSource* x);
// One product of many tokens by few weights, which quantises the tokens (row by row) itself.
bool narrow_layer(int64_t m, int64_t n, int64_t k);
void product_narrow(Ctx& c, const Product& p, const QuantSource& x);
void fill_zero(Ctx& c, float* p, int64_t rows, int64_t cols, int64_t pitch);

// ------------------------------------------------------------------ optimiser
struct AdamwConstants { float beta1, beta2, one_minus_beta1, one_minus_beta2, eps, step_scale, inv_sqrt_bc2, grad_scale, max_norm; };
int64_t adamw_norm_parts(const st_adamw_tensor* t, int n);
void adamw_step(Ctx& c, const st_adamw_tensor* t, int n, const st_adamw_opts& o, const AdamwConstants& k, char* workspace);
void adamw_state(Ctx& c, const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n, float* m_out, float* v_out);

}  // namespace st
