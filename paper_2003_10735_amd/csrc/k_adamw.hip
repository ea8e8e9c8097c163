// AdamW over a list of tensors.  A launch takes up to ST_ADAMW_PER_LAUNCH tensors, whose pointers travel with its arguments; every block
// takes one tile of one of them.
#include "st_dense.hpp"

namespace st {

constexpr int TILE = 2048;                 // values a block of 256 threads
constexpr float TINY = 0x1p-100f;          // a run of an 8-bit state whose largest value is less holds zeros

struct TensorRef { void* p; const void* g; void* m; void* v; float* ms; float* vs; void* copy; long long n; };
struct TensorList {
    TensorRef t[ST_ADAMW_PER_LAUNCH];
    float decay[ST_ADAMW_PER_LAUNCH];      // 1 - lr * weight_decay
    unsigned first[ST_ADAMW_PER_LAUNCH + 1];   // first tile of each
    int n;
};
static_assert(sizeof(TensorList) + sizeof(AdamwConstants) + 64 <= 4096, "kernel arguments");

__device__ __forceinline__ int tensor_of(const TensorList& l, unsigned tile)
{
    int lo = 0, hi = l.n - 1;              // the last tensor that begins at or before the tile (tensors without values own no tile)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (l.first[mid] <= tile) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Four consecutive values from p + i, of which `n` exist (the others are 0).
template <class T> __device__ __forceinline__ void load4(const T* p, int n, bool wide, float (&v)[4])
{
    if (wide && n >= 4) {
        if (sizeof(T) == 2) {
            const uint2 u = *(const uint2*)p;
            v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
            v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
        } else {
            const float4 u = *(const float4*)p;
            v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
}
template <class T> __device__ __forceinline__ void store4(T* p, int n, bool wide, const float (&v)[4])
{
    if (wide && n >= 4) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        *(T4*)p = T4{from_f32<T>(v[0]), from_f32<T>(v[1]), from_f32<T>(v[2]), from_f32<T>(v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < n) p[i] = from_f32<T>(v[i]);
}
__device__ __forceinline__ bool aligned(const void* p, unsigned bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// ------------------------------------------------------------------------------------------------------ norm
// Squares and their sums in float64: no gradient that is finite makes the norm infinite, and the order of the sums does not show.
template <class G>
__global__ __launch_bounds__(256) void k_grad_square_sums(const TensorList l, float grad_scale, double* __restrict__ parts)
{
    __shared__ double sums[4];
    const int i = tensor_of(l, blockIdx.x);
    const G* g = (const G*)l.t[i].g;
    const long long n = l.t[i].n, base = (long long)(blockIdx.x - l.first[i]) * TILE;
    const bool wide = aligned(g, 4 * sizeof(G));
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < TILE / 1024; ++j) {
        const long long at = base + j * 1024 + threadIdx.x * 4;
        if (at >= n) break;
        float v[4];
        load4(g + at, n - at < 4 ? (int)(n - at) : 4, wide, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) { const double d = (double)(v[k] * grad_scale); s += d * d; }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) parts[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}
__global__ __launch_bounds__(1024) void k_norm(const double* __restrict__ parts, long long n, float* __restrict__ norm, float* __restrict__ out)
{
    __shared__ double sums[16];
    double s = 0.0;
    for (long long i = threadIdx.x; i < n; i += 1024) s += parts[i];
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int i = 0; i < 16; ++i) s += sums[i];
        const float v = (float)sqrt(s);
        *norm = v;
        if (out) *out = v;
    }
}

// ------------------------------------------------------------------------------------------------------ step
// The factor on the gradients, or 0 where the step is not taken (grad_scale and max_norm are positive).
__device__ __forceinline__ float clip_factor(const AdamwConstants& k, const float* norm)
{
    if (!norm) return k.grad_scale;
    const float v = *norm;
    if (!(v < __builtin_inff())) return 0.f;
    return v > k.max_norm ? k.grad_scale * (k.max_norm / v) : k.grad_scale;
}
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = max(v, (unsigned)__shfl_xor((int)v, d));
    return v;
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

// One tile.  A lane takes four neighbouring values of a run of 256, a wavefront a run at a time.  Every operation is a float32 operation
// of its own (no fused ones), in the order of the header's formulas: codes change by whole steps, so two programs that are to give the
// same codes have to round alike.
template <class P, class G, int BITS>
__global__ __launch_bounds__(256) void k_adamw(const TensorList l, const AdamwConstants k, const float* __restrict__ norm)
{
    const int i = tensor_of(l, blockIdx.x);
    const TensorRef t = l.t[i];
    const float decay = l.decay[i], factor = clip_factor(k, norm);
    if (factor == 0.f) return;
    P* pp = (P*)t.p;
    const G* gg = (const G*)t.g;
    const bool wp = aligned(pp, 4 * sizeof(P)), wg = aligned(gg, 4 * sizeof(G)), wc = aligned(t.copy, 8);
    const bool wm = aligned(t.m, BITS == 8 ? 4 : 16) && aligned(t.v, BITS == 8 ? 4 : 16);
    const long long base = (long long)(blockIdx.x - l.first[i]) * TILE;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int j = 0; j < TILE / 1024; ++j) {
        const long long run = base + (j * 4 + wave) * 256, at = run + lane * 4;
        if (run >= t.n) break;
        const int n = t.n - at >= 4 ? 4 : t.n - at > 0 ? (int)(t.n - at) : 0;
        float p[4], g[4], m[4], v[4], u[4];
        load4(pp + at, n, wp, p);
        load4(gg + at, n, wg, g);
        if constexpr (BITS == 32) {
            load4((const float*)t.m + at, n, wm, m);
            load4((const float*)t.v + at, n, wm, v);
        } else {
            const float ms = t.ms[run / 256], vs = t.vs[run / 256];
            unsigned cm = 0, cv = 0;
            if (wm && n == 4) { cm = *(const unsigned*)((const char*)t.m + at); cv = *(const unsigned*)((const char*)t.v + at); }
            else for (int e = 0; e < n; ++e) {
                cm |= (unsigned)((const uint8_t*)t.m)[at + e] << (8 * e);
                cv |= (unsigned)((const uint8_t*)t.v)[at + e] << (8 * e);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float qm = (float)(int8_t)(cm >> (8 * e)), qv = (float)(uint8_t)(cv >> (8 * e));
                m[e] = qm * fabsf(qm) * ms;
                const float root = qv * qv * vs;
                v[e] = root * root;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = g[e] * factor;
            m[e] = m[e] * k.beta1 + ge * k.one_minus_beta1;
            v[e] = v[e] * k.beta2 + ge * ge * k.one_minus_beta2;
            u[e] = sqrtf(v[e]);
            p[e] = p[e] * decay - k.step_scale * (m[e] / (u[e] * k.inv_sqrt_bc2 + k.eps));
        }
        store4(pp + at, n, wp, p);
        if (t.copy) store4((bf16*)t.copy + at, n, wc, p);
        if constexpr (BITS == 32) {
            store4((float*)t.m + at, n, wm, m);
            store4((float*)t.v + at, n, wm, v);
        } else {
            unsigned tm = 0, tv = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) { tm = max(tm, __float_as_uint(m[e]) & 0x7fffffffu); tv = max(tv, __float_as_uint(u[e]) & 0x7fffffffu); }
            tm = wave_max(tm); tv = wave_max(tv);
            float ms, vs;
            const float rm = run_multiplier(tm, 16129.f, &ms), rv = run_multiplier(tv, 65025.f, &vs);
            if (lane == 0) { t.ms[run / 256] = ms; t.vs[run / 256] = vs; }
            unsigned cm = 0, cv = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                int qm = rm == 0.f ? 0 : (int)rintf(sqrtf(fabsf(m[e]) * rm));
                if (m[e] < 0.f) qm = -qm;
                int qv = rv == 0.f ? 0 : (int)rintf(sqrtf(u[e] * rv));
                if (rv != 0.f && qv == 0 && u[e] > 0.f) qv = 1;
                cm |= (unsigned)(uint8_t)qm << (8 * e);
                cv |= (unsigned)(uint8_t)qv << (8 * e);
            }
            if (wm && n == 4) { *(unsigned*)((char*)t.m + at) = cm; *(unsigned*)((char*)t.v + at) = cv; }
            else for (int e = 0; e < n; ++e) {
                ((uint8_t*)t.m)[at + e] = (uint8_t)(cm >> (8 * e));
                ((uint8_t*)t.v)[at + e] = (uint8_t)(cv >> (8 * e));
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------------ state's values
__global__ __launch_bounds__(256) void k_adamw_state(const int8_t* __restrict__ m, const float* __restrict__ ms, const uint8_t* __restrict__ v,
                                                     const float* __restrict__ vs, long long n, float* __restrict__ m_out, float* __restrict__ v_out)
{
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= n) return;
    const int cnt = n - at >= 4 ? 4 : (int)(n - at);
    const bool whole = cnt == 4;
    if (m_out) {
        const float s = ms[at / 256];
        float o[4];
        const bool wide = whole && aligned(m, 4);
        const unsigned c = wide ? *(const unsigned*)(m + at) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float q = (float)(wide ? (int8_t)(c >> (8 * e)) : e < cnt ? m[at + e] : (int8_t)0);
            o[e] = q * fabsf(q) * s;
        }
        store4(m_out + at, cnt, aligned(m_out, 16), o);
    }
    if (v_out) {
        const float s = vs[at / 256];
        float o[4];
        const bool wide = whole && aligned(v, 4);
        const unsigned c = wide ? *(const unsigned*)(v + at) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float q = (float)(wide ? (uint8_t)(c >> (8 * e)) : e < cnt ? v[at + e] : (uint8_t)0);
            const float root = q * q * s;
            o[e] = root * root;
        }
        store4(v_out + at, cnt, aligned(v_out, 16), o);
    }
}

// ------------------------------------------------------------------------------------------------------ host
int64_t adamw_tiles(const st_adamw_tensor* t, int n)
{
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) tiles += ceil_div(t[i].n, TILE);
    return tiles;
}

// Calls f(list, tiles) for the list in pieces that a launch can take.
template <class F> static void for_pieces(const st_adamw_tensor* t, int n, double lr, F f)
{
    for (int at = 0; at < n;) {
        TensorList l;
        l.n = 0;
        l.first[0] = 0;
        int64_t tiles = 0;
        for (; at < n && l.n < ST_ADAMW_PER_LAUNCH; ++at) {
            if (t[at].n == 0) continue;
            const int64_t more = ceil_div(t[at].n, TILE);
            if (l.n && tiles + more > 0x7fffffff) break;
            l.t[l.n] = TensorRef{t[at].param, t[at].grad, t[at].m, t[at].v, t[at].m_scale, t[at].v_scale, t[at].copy, t[at].n};
            l.decay[l.n] = (float)(1.0 - lr * t[at].weight_decay);
            tiles += more;
            l.first[++l.n] = (unsigned)tiles;
        }
        if (l.n) f(l, (unsigned)tiles);
    }
}

void adamw_norm(Ctx& c, const st_adamw_tensor* t, int n, int grad_bf16, float grad_scale, double* parts, float* norm, float* out)
{
    int64_t done = 0;
    for_pieces(t, n, 0.0, [&](const TensorList& l, unsigned tiles) {
        if (grad_bf16) ST_LAUNCH(c, "grad_square_sums", k_grad_square_sums<bf16>, dim3(tiles), dim3(256), 0, l, grad_scale, parts + done);
        else           ST_LAUNCH(c, "grad_square_sums", k_grad_square_sums<float>, dim3(tiles), dim3(256), 0, l, grad_scale, parts + done);
        done += tiles;
    });
    ST_LAUNCH(c, "grad_norm", k_norm, dim3(1), dim3(1024), 0, parts, (long long)done, norm, out);
}

template <class P, class G, int BITS>
static void step(Ctx& c, const st_adamw_tensor* t, int n, double lr, const AdamwConstants& k, const float* norm)
{
    for_pieces(t, n, lr, [&](const TensorList& l, unsigned tiles) {
        ST_LAUNCH(c, "adamw", (k_adamw<P, G, BITS>), dim3(tiles), dim3(256), 0, l, k, norm);
    });
}

// norm: clip by it; null: do not
void adamw_step(Ctx& c, const st_adamw_tensor* t, int n, const st_adamw_opts& o, const AdamwConstants& k, const float* norm)
{
#define ST_STEP(P, G)                                                  \
    do {                                                               \
        if (o.state_bits == 8) step<P, G, 8>(c, t, n, o.lr, k, norm);  \
        else step<P, G, 32>(c, t, n, o.lr, k, norm);                   \
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
