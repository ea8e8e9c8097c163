// AdamW over a list of tensors.  A launch takes up to ST_ADAMW_PER_LAUNCH tensors, whose pointers travel with its arguments; every block
// takes one tile of one of them.
#include "st_lists.hpp"
#include "st_quantize.hpp"

#include <algorithm>

namespace st {

// Values a block of 256 threads steps: runs of 256 a wavefront, two with states in 8 bits, one with 32 (77 M values with states in 32 bits,
// the whole call, 435 us with 1024, 447 with 2048, 459 with 4096; 436 M with 8 bits 2112, 2032, 2093).
constexpr int tile_of(int bits) { return bits == 8 ? 2048 : 1024; }
constexpr int NORM_BLOCKS = 2048, NORM_PER_LAUNCH = 160;
// values of a tile of the norm: small lists are spread over more blocks
static int norm_tile(int64_t all) { return all <= (int64_t)NORM_BLOCKS * 2048 ? 2048 : 8192; }
constexpr float TINY = 0x1p-100f;          // a run of an 8-bit state whose largest value is less holds zeros

struct TensorRef { void* p; const void* g; void* m; void* v; float* ms; float* vs; void* copy; long long n; };
struct TensorList {
    TensorRef t[ST_ADAMW_PER_LAUNCH];
    float decay[ST_ADAMW_PER_LAUNCH];      // 1 - lr * weight_decay
    unsigned first[ST_ADAMW_PER_LAUNCH + 1];   // first tile of each
    int n;
};
struct GradList {
    const void* g[NORM_PER_LAUNCH]; long long n[NORM_PER_LAUNCH];
    unsigned first[NORM_PER_LAUNCH + 1];
    int count;
};
static_assert(sizeof(TensorList) + sizeof(AdamwConstants) + 64 <= 4096 && sizeof(GradList) + 64 <= 4096, "kernel arguments");

// What a step writes is read by the next one: its stores do not ask for room in L2.
template <class T> __device__ __forceinline__ void store4(T* p, int n, const float (&v)[4])
{
    if (n >= 4) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        typedef T4 T4any __attribute__((aligned(sizeof(T))));
        __builtin_nontemporal_store(T4{from_f32<T>(v[0]), from_f32<T>(v[1]), from_f32<T>(v[2]), from_f32<T>(v[3])}, (T4any*)p);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < n) p[i] = from_f32<T>(v[i]);
}
// four codes, of which `n` exist
template <bool NT = false> __device__ __forceinline__ unsigned load_codes(const void* p, int n)
{
    if (n >= 4) return ST_LOAD(NT, u32_1, p);
    unsigned c = 0;
    for (int e = 0; e < n; ++e) c |= (unsigned)((const uint8_t*)p)[e] << (8 * e);
    return c;
}
// Codes are stored past L2 where the list is streamed: 436 M values, 1843 us a step and the reading of its state with, 1914 without; 24 heads,
// not streamed, 73.4 and 72.1.  (One tensor of 100 M values: 267 and 259; with codes one byte off their line 341 and 282.)
template <bool NT = false> __device__ __forceinline__ void store_codes(void* p, int n, unsigned c)
{
    if (n >= 4) {
        if constexpr (NT) __builtin_nontemporal_store(c, (u32_1*)p);
        else *(u32_1*)p = c;
        return;
    }
    for (int e = 0; e < n; ++e) ((uint8_t*)p)[e] = (uint8_t)(c >> (8 * e));
}

// ------------------------------------------------------------------------------------------------------ norm
// Squares and their sums in float64: no square of a finite gradient is infinite, and the order of the sums does not show.  A
// launch has NORM_BLOCKS blocks at most, so that few parts are left to be added.  Bytes bound it: 436 M bfloat16 values in 146 us, 6.0 TB/s.
template <class G, int RUNS>
__global__ __launch_bounds__(256) void k_grad_square_sums(const GradList l, float grad_scale, unsigned tiles, double* __restrict__ parts)
{
    __shared__ double sums[4];
    // a block's tiles follow one another, so that the tensor is searched once
    const unsigned each = tiles / gridDim.x, rest = tiles - each * gridDim.x;
    unsigned tile = blockIdx.x * each + min(blockIdx.x, rest);
    const unsigned end = tile + each + (blockIdx.x < rest ? 1 : 0);
    int i = tensor_of<NORM_PER_LAUNCH>(l.first, l.count, tile);
    double s = 0.0;
    for (; tile < end; ++tile) {
        while (i + 1 < l.count && tile >= l.first[i + 1]) ++i;
        const G* g = (const G*)l.g[i];
        const long long base = (long long)(tile - l.first[i]) * (RUNS * 2048) + threadIdx.x * 8;
        Raw8<G> v[RUNS];
        load_row(g, l.n[i], [&](int j) { return base + j * 2048; }, v);
#pragma unroll
        for (int j = 0; j < RUNS; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) { const double d = (double)(v[j][k] * grad_scale); s = __builtin_fma(d, d, s); }
    }
    s = block_sum(s, sums);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}
__device__ __forceinline__ float norm_of_parts(const double* __restrict__ parts, int n, double* sums)
{
    double s = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) s += parts[i];
    return (float)sqrt(block_sum(s, sums));
}
__global__ __launch_bounds__(256) void k_norm(const double* __restrict__ parts, int n, float* __restrict__ norm, float* __restrict__ out)
{
    __shared__ double sums[4];
    const float v = norm_of_parts(parts, n, sums);
    if (threadIdx.x == 0) { *norm = v; if (out) *out = v; }
}

// ------------------------------------------------------------------------------------------------------ step
// The norm, as it reaches a step: a value, or (parts > 0) the parts of it, which every block of a small launch adds by itself; the first
// block then also writes it to `out`.
struct NormRef { const float* norm; const double* parts; int n_parts; float* out; };

// The factor on the gradients, or -1 where the step is not taken (grad_scale and max_norm are positive; their product may vanish).
__device__ __forceinline__ float clip_factor(const AdamwConstants& k, float norm)
{
    if (!(norm < __builtin_inff())) return -1.f;
    return norm > k.max_norm ? k.grad_scale * (k.max_norm / norm) : k.grad_scale;
}
// scale and multiplier of a run whose largest value has the bits `top`; codes^2 reach `codes2`
__device__ __forceinline__ float run_multiplier(unsigned top, float codes2, float* scale)
{
    const float a = __uint_as_float(top);
    if (a < TINY) { *scale = 0.f; return 0.f; }
    if (top >= 0x7f800000u) { *scale = __uint_as_float(0x7fc00000u); return 0.f; }   // infinity or NaN
    *scale = a * (1.f / codes2);
    return codes2 * (1.f / a);
}
// Square root, rounded to the nearest float32, of 0 and of normal numbers from 2^-96 on (and of infinity and NaN), by Tuckerman's rounding
// test.  The instruction's result s is off by one unit in the last place at most; s (s +- unit) is s^2 beyond the middle between the two candidates, so the sign of
// its difference from x, which a fused multiply-add has exactly, decides.
__device__ __forceinline__ float sqrt_rn(float x)
{
    const float s = __builtin_amdgcn_sqrtf(x);
    const float lo = __uint_as_float(__float_as_uint(s) - 1), hi = __uint_as_float(__float_as_uint(s) + 1);
    const float r_lo = __builtin_fmaf(-lo, s, x), r_hi = __builtin_fmaf(-hi, s, x);
    const float t = r_lo <= 0.f ? lo : s;
    return r_hi > 0.f ? hi : t;
}
constexpr unsigned SQRT_LEAST = 0x0f800000u;      // 2^-96
constexpr float ROUND = 12582912.f;               // 1.5 * 2^23: a sum with it ends in the other number's nearest whole number, low byte first

// Codes of four values: their shares y times the sign of `of`, as four bytes.  The instruction's root settles the whole number unless it
// lies next to a middle, which one look at all four finds out.  A value that is no number, or a share of one, gets the byte 0.
__device__ __forceinline__ unsigned codes_of(const float (&y)[4], const float (&of)[4], const float (&least)[4])
{
    float t[4], off = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float s = __builtin_copysignf(fmaxf(__builtin_amdgcn_sqrtf(y[e]), least[e]), of[e]);
        t[e] = s + ROUND;
        off = fmaxf(off, fabsf(s - (t[e] - ROUND)));
    }
    if (off > 0.4999f)
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = __builtin_copysignf(fmaxf(sqrt_rn(y[e]), least[e]), of[e]) + ROUND;
    return pack4(__float_as_uint(t[0]), __float_as_uint(t[1]), __float_as_uint(t[2]), __float_as_uint(t[3]));
}

// One tile.  A lane takes four neighbouring values of a run of 256, a wavefront one or two runs, whose loads are all under way before the
// first is used.  What the codes depend on is float32 operations of their own (no fused ones), in the order of the header's formulas:
// codes change by whole steps, so two programs that are to give the same codes have to round alike.  The parameters' quotient is a
// product with a reciprocal of one unit's accuracy.
// STREAM: the list is more than the cache behind L2 holds, and its loads do not ask for room either.
// Bytes bound it, and with states in 8 bits about as much the arithmetic of the codes: 77.6 M values, 32 bits, 345 us, 5.8 TB/s; 436 M values,
// 8 bits, bfloat16 gradients, 980 us, 6.2 TB/s at 94 % busy vector units.
template <class P, class G, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void k_adamw(const TensorList l, const AdamwConstants k, const NormRef nr)
{
    constexpr int RUNS = tile_of(BITS) / 1024;
    __shared__ double sums[4];
    const int i = tensor_of<ST_ADAMW_PER_LAUNCH>(l.first, l.n, blockIdx.x);
    const TensorRef& t = l.t[i];
    P* pp = (P*)t.p;
    const G* gg = (const G*)t.g;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long base = (long long)(blockIdx.x - l.first[i]) * tile_of(BITS) + wave * (RUNS * 256);
    float p[RUNS][4], g[RUNS][4], m[RUNS][4], v[RUNS][4], ms[RUNS], vs[RUNS];
    unsigned cm[RUNS], cv[RUNS];
    int n[RUNS];
#pragma unroll
    for (int j = 0; j < RUNS; ++j) {
        const long long run = base + j * 256, at = run + lane * 4;
        n[j] = t.n - at >= 4 ? 4 : t.n - at > 0 ? (int)(t.n - at) : 0;
        load4<STREAM>(pp + at, n[j], p[j]);
        load4<STREAM>(gg + at, n[j], g[j]);
        if constexpr (BITS == 32) {
            load4<STREAM>((const float*)t.m + at, n[j], m[j]);
            load4<STREAM>((const float*)t.v + at, n[j], v[j]);
        } else {
            ms[j] = vs[j] = 0.f;
            if (run < t.n) { ms[j] = t.ms[run / 256]; vs[j] = t.vs[run / 256]; }
            cm[j] = load_codes<STREAM>((const char*)t.m + at, n[j]); cv[j] = load_codes<STREAM>((const char*)t.v + at, n[j]);
        }
    }
    float factor = k.grad_scale;
    if (nr.norm || nr.parts) {
        const float norm = nr.parts ? norm_of_parts(nr.parts, nr.n_parts, sums) : *nr.norm;
        if (nr.parts && nr.out && blockIdx.x == 0 && threadIdx.x == 0) *nr.out = norm;
        factor = k.max_norm > 0.f ? clip_factor(k, norm) : k.grad_scale;
        if (factor < 0.f) return;
    }
    const float decay = l.decay[i];
#pragma unroll
    for (int j = 0; j < RUNS; ++j) {
        const long long run = base + j * 256, at = run + lane * 4;
        if (run >= t.n) break;
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BITS == 8) {
                const float qm = (float)(int8_t)(cm[j] >> (8 * e)), qv = (float)(uint8_t)(cv[j] >> (8 * e));
                m[j][e] = qm * fabsf(qm) * ms[j];
                const float root = qv * qv * vs[j];
                v[j][e] = root * root;
            }
            const float ge = g[j][e] * factor;
            m[j][e] = m[j][e] * k.beta1 + ge * k.one_minus_beta1;
            v[j][e] = v[j][e] * k.beta2 + ge * ge * k.one_minus_beta2;
            u[e] = BITS == 8 ? sqrt_rn(v[j][e]) : sqrtf(v[j][e]);
        }
        if constexpr (BITS == 8) {
            unsigned least = 0xffffffffu;      // (0 is none of the small ones)
#pragma unroll
            for (int e = 0; e < 4; ++e) least = min(least, __float_as_uint(v[j][e]) - 1);
            if (least < SQRT_LEAST - 1)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = sqrtf(v[j][e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            p[j][e] = __builtin_fmaf(-k.step_scale, m[j][e] * __builtin_amdgcn_rcpf(__builtin_fmaf(u[e], k.inv_sqrt_bc2, k.eps)), p[j][e] * decay);
        store4(pp + at, n[j], p[j]);
        if (t.copy) store4((bf16*)t.copy + at, n[j], p[j]);
        if constexpr (BITS == 32) {
            store4((float*)t.m + at, n[j], m[j]);
            store4((float*)t.v + at, n[j], v[j]);
        } else {
            // (values that do not exist are zeros: their gradient and state were)
            const unsigned tm = max(max(abs_bits(m[j][0]), abs_bits(m[j][1])), max(abs_bits(m[j][2]), abs_bits(m[j][3])));
            const unsigned tv = max(max(__float_as_uint(u[0]) & ABS_BITS, __float_as_uint(u[1]) & ABS_BITS),
                                    max(__float_as_uint(u[2]) & ABS_BITS, __float_as_uint(u[3]) & ABS_BITS));
            float new_ms, new_vs;
            const float rm = run_multiplier(wave_max(tm), 16129.f, &new_ms), rv = run_multiplier(wave_max(tv), 65025.f, &new_vs);
            if (lane == 0) { t.ms[run / 256] = new_ms; t.vs[run / 256] = new_vs; }
            const float one = rv == 0.f ? 0.f : 1.f;
            float ym[4], yv[4], none[4], some[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ym[e] = fabsf(m[j][e]) * rm; none[e] = 0.f;
                yv[e] = u[e] * rv; some[e] = u[e] > 0.f ? one : 0.f;
            }
            const unsigned qm = codes_of(ym, m[j], none), qv = codes_of(yv, u, some);
            store_codes<STREAM>((char*)t.m + at, n[j], qm); store_codes<STREAM>((char*)t.v + at, n[j], qv);
        }
    }
}

// ------------------------------------------------------------------------------------------------------ state's values
// Bytes bound it: 436 M values, both kinds, 726 us, 6.0 TB/s.
__global__ __launch_bounds__(256) void k_adamw_state(const int8_t* __restrict__ m, const float* __restrict__ ms, const uint8_t* __restrict__ v,
                                                     const float* __restrict__ vs, long long n, float* __restrict__ m_out, float* __restrict__ v_out)
{
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= n) return;
    const int count = n - at >= 4 ? 4 : (int)(n - at);
    float o[4];
    if (m_out) {
        const float s = ms[at / 256];
        const unsigned c = load_codes(m + at, count);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float q = (float)(int8_t)(c >> (8 * e));
            o[e] = q * fabsf(q) * s;
        }
        store4(m_out + at, count, o);
    }
    if (v_out) {
        const float s = vs[at / 256];
        const unsigned c = load_codes(v + at, count);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float q = (float)(uint8_t)(c >> (8 * e)), root = q * q * s;
            o[e] = root * root;
        }
        store4(v_out + at, count, o);
    }
}

// ------------------------------------------------------------------------------------------------------ host
// The gradients in pieces that a launch of the norm can take: f(list, tiles).
template <class F> static void for_grads(const st_adamw_tensor* t, int n, F f)
{
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += t[i].n;
    const int tile = norm_tile(all);
    for (int at = 0; at < n;) {
        GradList l;
        l.count = 0;
        l.first[0] = 0;
        int64_t tiles = 0;
        for (; at < n && l.count < NORM_PER_LAUNCH; ++at) {
            if (t[at].n == 0) continue;
            const int64_t more = ceil_div(t[at].n, tile);
            if (l.count && tiles + more > 0xffffff) break;
            l.g[l.count] = t[at].grad;
            l.n[l.count] = t[at].n;
            tiles += more;
            l.first[++l.count] = (unsigned)tiles;
        }
        if (l.count) f(l, (unsigned)tiles, tile);
    }
}
int64_t adamw_norm_parts(const st_adamw_tensor* t, int n)
{
    int64_t parts = 0;
    for_grads(t, n, [&](const GradList&, unsigned tiles, int) { parts += std::min<unsigned>(tiles, NORM_BLOCKS); });
    return parts;
}
// Calls f(list, tiles) for the list in pieces that a launch can take.
template <class F> static void for_pieces(const st_adamw_tensor* t, int n, double lr, int tile, F f)
{
    for (int at = 0; at < n;) {
        TensorList l;
        l.n = 0;
        l.first[0] = 0;
        int64_t tiles = 0;
        for (; at < n && l.n < ST_ADAMW_PER_LAUNCH; ++at) {
            if (t[at].n == 0) continue;
            const int64_t more = ceil_div(t[at].n, tile);
            if (l.n && tiles + more > 0xffffff) break;
            l.t[l.n] = TensorRef{t[at].param, t[at].grad, t[at].m, t[at].v, t[at].m_scale, t[at].v_scale, t[at].copy, t[at].n};
            l.decay[l.n] = (float)(1.0 - lr * t[at].weight_decay);
            tiles += more;
            l.first[++l.n] = (unsigned)tiles;
        }
        if (l.n) f(l, (unsigned)tiles);
    }
}

template <class P, class G, int BITS>
static void step(Ctx& c, const st_adamw_tensor* t, int n, double lr, const AdamwConstants& k, bool stream, NormRef nr)
{
    for_pieces(t, n, lr, tile_of(BITS), [&](const TensorList& l, unsigned tiles) {
        if (stream) ST_LAUNCH(c, "adamw", (k_adamw<P, G, BITS, true>), dim3(tiles), dim3(256), 0, l, k, nr);
        else ST_LAUNCH(c, "adamw", (k_adamw<P, G, BITS, false>), dim3(tiles), dim3(256), 0, l, k, nr);
        nr.out = nullptr;
    });
}

// workspace: the norm and, 256 bytes on, its parts; null: no norm
void adamw_step(Ctx& c, const st_adamw_tensor* t, int n, const st_adamw_opts& o, const AdamwConstants& k, char* workspace)
{
    NormRef nr{nullptr, nullptr, 0, nullptr};
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) tiles += ceil_div(t[i].n, tile_of(o.state_bits));
    if (workspace) {
        double* parts = (double*)(workspace + 256);
        int done = 0;
        for_grads(t, n, [&](const GradList& l, unsigned norm_tiles, int tile) {
            const unsigned blocks = std::min<unsigned>(norm_tiles, NORM_BLOCKS);
#define ST_SUMS(G, RUNS)                                                                                                          \
    ST_LAUNCH(c, "grad_square_sums", (k_grad_square_sums<G, RUNS>), dim3(blocks), dim3(256), 0, l, k.grad_scale, norm_tiles, parts + done)
            if (o.grad_dtype == ST_BF16) { if (tile == 2048) ST_SUMS(bf16, 1); else ST_SUMS(bf16, 4); }
            else                         { if (tile == 2048) ST_SUMS(float, 1); else ST_SUMS(float, 4); }
#undef ST_SUMS
            done += (int)blocks;
        });
        // Up to some 2000 tiles the step adds the parts itself, every block all of them; beyond, that costs more than a launch of its own.  Lists
        // of heads, us a call, added in each block and by a launch: 32 bits, 438 tiles 8.5 and 9.8, 1752 12.8 and 14.3, 2190 17.9 and 18.7, 2628
        // 20.4 and 20.5, 3942 32.7 and 30.5; 8 bits, 884 tiles 13.1 and 14.4, 1768 18.1 and 18.9, 2210 29.1 and 28.9, 3978 45.8 and 44.7.
        if (tiles > 0 && tiles <= 2048 && done <= NORM_BLOCKS) nr = NormRef{nullptr, parts, done, o.grad_norm};
        else {
            ST_LAUNCH(c, "grad_norm", k_norm, dim3(1), dim3(256), 0, parts, done, (float*)workspace, o.grad_norm);
            nr.norm = (const float*)workspace;
        }
    }
    if (tiles == 0) return;
    // One list stepped again and again, us a step with plain loads and with these: heads of 445 075 values, states in 32 bits, 24 of them
    // (171 MB) 65 and 68, 48 (342 MB) 153 and 136, 200 683 and 566; in 8 bits, 48 (214 MB) 106 and 106, 96 (428 MB) 244 and 211.
    const int64_t each = (o.param_dtype == ST_BF16 ? 2 : 4) + (o.grad_dtype == ST_BF16 ? 2 : 4) + (o.state_bits == 8 ? 2 : 8);
    int64_t values = 0;
    for (int i = 0; i < n; ++i) values += t[i].n;
    const bool stream = values * each > (int64_t)256 << 20;
#define ST_STEP(P, G)                                                  \
    do {                                                               \
        if (o.state_bits == 8) step<P, G, 8>(c, t, n, o.lr, k, stream, nr);    \
        else step<P, G, 32>(c, t, n, o.lr, k, stream, nr);                     \
    } while (0)
    if (o.param_dtype == ST_F32) { if (o.grad_dtype == ST_F32) ST_STEP(float, float); else ST_STEP(float, bf16); }
    else                         { if (o.grad_dtype == ST_F32) ST_STEP(bf16, float); else ST_STEP(bf16, bf16); }
#undef ST_STEP
}

void adamw_state(Ctx& c, const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n, float* m_out, float* v_out)
{
    ST_LAUNCH(c, "adamw_state", k_adamw_state, dim3((unsigned)ceil_div(n, 1024)), dim3(256), 0, m, m_scale, v, v_scale, (long long)n, m_out, v_out);
}

}  // namespace st
