// Codes and scales of rows, for the kernels that quantise (k_quantize.hip says what is computed).
#pragma once
#include "st_dense.hpp"

namespace st {

constexpr unsigned ABS_BITS = 0x7fffffffu, INF_BITS = 0x7f800000u;
constexpr unsigned SMALLEST_TOP = 0x04000000u;     // 2^-119: 127 / a is finite from 2^-121 on

__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & ABS_BITS; }

// multiplier and scale of a row whose largest |value| has the bits `top`
__device__ __forceinline__ float row_multiplier(unsigned top, float* scale)
{
    if (top < SMALLEST_TOP) { *scale = 0.f; return 0.f; }
    if (top >= INF_BITS) { *scale = __uint_as_float(0x7fc00000u); return 0.f; }
    const float a = __uint_as_float(top);
    *scale = a * (1.f / 127.f);
    return 127.f * (1.f / a);
}
// the code in the low byte; a multiplier of 0 stands for a row of zeros or of no numbers, whose codes are 0 whatever v is
__device__ __forceinline__ unsigned code_of(float v, float r) { return r == 0.f ? 0u : __float_as_uint(v * r + 12582912.f); }
__device__ __forceinline__ unsigned pack4(unsigned a, unsigned b, unsigned c, unsigned d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}

// largest of a wavefront's values, in a scalar register: four steps inside rows of 16 lanes, two across
#define ST_DPP(CTRL, ROWS) v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false))
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    ST_DPP(0x111, 0xf); ST_DPP(0x112, 0xf); ST_DPP(0x114, 0xf); ST_DPP(0x118, 0xf);      // row_shr 1, 2, 4, 8
    ST_DPP(0x142, 0xa); ST_DPP(0x143, 0xc);                                              // row_bcast 15, 31
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
// .. of each half of a wavefront's lanes
__device__ __forceinline__ unsigned half_max(unsigned v)
{
    ST_DPP(0x111, 0xf); ST_DPP(0x112, 0xf); ST_DPP(0x114, 0xf); ST_DPP(0x118, 0xf);
    ST_DPP(0x142, 0xa);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)v, 31), hi = (unsigned)__builtin_amdgcn_readlane((int)v, 63);
    return threadIdx.x & 32 ? hi : lo;
}
#undef ST_DPP

// Several values at once, from or to any address that is a multiple of their own size: the card splits what is not aligned.  (Rows with an
// odd pitch value by value took 1.7 times as long: 5480 tokens 532 -> 6367.)
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_2 __attribute__((aligned(2)));
typedef u32x2 u32x2_2 __attribute__((aligned(2)));
typedef f32x4_t f32x4_4 __attribute__((aligned(4)));
typedef unsigned u32_1 __attribute__((aligned(1)));

// A load of what is not read again soon, past the caches' order of use (NT), or a plain one.  (A macro: a template would lose the type's
// alignment.)
#define ST_LOAD(NT, TYPE, P) ((NT) ? __builtin_nontemporal_load((const TYPE*)(P)) : *(const TYPE*)(P))

// Four consecutive values from p, of which `n` exist; the others are 0.
template <bool NT = false> __device__ __forceinline__ void load4(const bf16* p, int n, float (&v)[4])
{
    if (n >= 4) {
        const u32x2 w = ST_LOAD(NT, u32x2_2, p);
        v[0] = __uint_as_float(w[0] << 16); v[1] = __uint_as_float(w[0] & 0xffff0000u);
        v[2] = __uint_as_float(w[1] << 16); v[3] = __uint_as_float(w[1] & 0xffff0000u);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? (float)p[i] : 0.f;
}
template <bool NT = false> __device__ __forceinline__ void load4(const float* p, int n, float (&v)[4])
{
    if (n >= 4) {
        const f32x4_t w = ST_LOAD(NT, f32x4_4, p);
        v[0] = w[0]; v[1] = w[1]; v[2] = w[2]; v[3] = w[3];
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : 0.f;
}

// V (4 or 8) consecutive values as they lie in memory.  The run at `at` of a row of `len` values that ends inside it is loaded from
// run_start(): the row's last V values, which down() then moves to their places, zeros behind them.  Rows of fewer than V values are
// loaded one by one (load_short).
template <int V, class I> __device__ __forceinline__ I run_start(I at, I len) { return at < len - V ? at : len - V; }
template <class T, int V> struct Run;
template <int V> struct Run<bf16, V> {
    unsigned w[V / 2];
    template <bool NT = false> __device__ __forceinline__ void load(const bf16* p)
    {
        if constexpr (V == 8) { const u32x4_t u = ST_LOAD(NT, u32x4_2, p); w[0] = u[0]; w[1] = u[1]; w[2] = u[2]; w[3] = u[3]; }
        else { const u32x2 u = ST_LOAD(NT, u32x2_2, p); w[0] = u[0]; w[1] = u[1]; }
    }
    __device__ __forceinline__ void load_short(const bf16* p, int n, int64_t step = 1)      // one by one, `step` apart
    {
        const unsigned short* u = (const unsigned short*)p;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const unsigned lo = 2 * i < n ? u[2 * i * step] : 0u, hi = 2 * i + 1 < n ? u[(2 * i + 1) * step] : 0u;
            w[i] = lo | hi << 16;
        }
    }
    __device__ __forceinline__ void down(int d)
    {
#pragma unroll
        for (int s = 1; s < V / 2; s *= 2)
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[i] = d & (2 * s) ? (i + s < V / 2 ? w[i + s] : 0u) : w[i];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const unsigned odd = w[i] >> 16 | (i + 1 < V / 2 ? w[i + 1] << 16 : 0u);
            w[i] = d >= V ? 0u : d & 1 ? odd : w[i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
    // what follows unpacks the values again, instead of keeping them unpacked all the time
    __device__ __forceinline__ void repack()
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm volatile("" : "+v"(w[i]));
    }
    __device__ __forceinline__ void clear(int i) { w[i >> 1] &= i & 1 ? 0x0000ffffu : 0xffff0000u; }
};
template <int V> struct Run<float, V> {
    float v[V];
    template <bool NT = false> __device__ __forceinline__ void load(const float* p)
    {
#pragma unroll
        for (int i = 0; i < V; i += 4) { const f32x4_t a = ST_LOAD(NT, f32x4_4, (p + i)); v[i] = a[0]; v[i + 1] = a[1]; v[i + 2] = a[2]; v[i + 3] = a[3]; }
    }
    __device__ __forceinline__ void load_short(const float* p, int n, int64_t step = 1)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < n ? p[i * step] : 0.f;
    }
    __device__ __forceinline__ void down(int d)
    {
#pragma unroll
        for (int s = 1; s < V; s *= 2)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = d & s ? (i + s < V ? v[i + s] : 0.f) : v[i];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = d >= V ? 0.f : v[i];
    }
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
    __device__ __forceinline__ void repack() {}
    __device__ __forceinline__ void clear(int i) { v[i] = 0.f; }
};
template <int V> struct Run<void, V> {};      // no mask
template <class T> using Raw8 = Run<T, 8>;

// COUNT runs of eight of a row, run i at at(i): all under way before one of them is moved.
template <bool NT = false, class T, int COUNT, class I, class F>
__device__ __forceinline__ void load_row(const T* row, I len, F at, Raw8<T> (&v)[COUNT])
{
    if (len < 8) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i].load_short(row + at(i), at(i) < len ? (int)(len - at(i)) : 0);
        return;
    }
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i].template load<NT>(row + run_start<8, I>(at(i), len));
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const I d = at(i) - (len - 8);
        if (d > 0) v[i].down(d < 8 ? (int)d : 8);
    }
}

}  // namespace st
