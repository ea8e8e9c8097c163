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

// COUNT consecutive values from p, of which `n` exist; the others are 0.  wide: p is aligned for loads of all of them.
template <class T, int COUNT> __device__ __forceinline__ void load_run(const T* p, int64_t n, bool wide, float (&v)[COUNT])
{
    if (wide && n >= COUNT) {
        if constexpr (sizeof(T) == 2) {
            typedef unsigned W __attribute__((ext_vector_type(COUNT / 2)));
            const W w = *(const W*)p;
#pragma unroll
            for (int i = 0; i < COUNT / 2; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; i += 4) {
                const float4 w = *(const float4*)(p + i);
                v[i] = w.x; v[i + 1] = w.y; v[i + 2] = w.z; v[i + 3] = w.w;
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
}

// Eight consecutive values as they lie in memory, those from n on zeros.  wide: loaded at once, and n is either 8 or more or 0 or less.
template <class T> struct Raw8;
template <> struct Raw8<bf16> {
    unsigned w[4];
    __device__ __forceinline__ void load(const bf16* p, int n, bool wide)
    {
        if (wide) { const uint4 u = n > 0 ? *(const uint4*)p : make_uint4(0, 0, 0, 0); w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; return; }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned lo = 2 * i < n ? ((const unsigned short*)p)[2 * i] : 0u, hi = 2 * i + 1 < n ? ((const unsigned short*)p)[2 * i + 1] : 0u;
            w[i] = lo | hi << 16;
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
    // what follows unpacks the values again, instead of keeping them unpacked all the time
    __device__ __forceinline__ void repack() { asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3])); }
    __device__ __forceinline__ void clear(int i) { w[i >> 1] &= i & 1 ? 0x0000ffffu : 0xffff0000u; }
};
template <> struct Raw8<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* p, int n, bool wide)
    {
        if (wide) {
            const float4 a = n > 0 ? ((const float4*)p)[0] : make_float4(0, 0, 0, 0), b = n > 0 ? ((const float4*)p)[1] : make_float4(0, 0, 0, 0);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
    __device__ __forceinline__ void repack() {}
    __device__ __forceinline__ void clear(int i) { v[i] = 0.f; }
};

inline bool wide_ok(const void* p, int64_t pitch, int is_bf16, int run)     // runs of `run` values can be loaded at once
{
    const int64_t e = is_bf16 ? 2 : 4, bytes = run * e < 16 ? run * e : 16;
    return (uintptr_t)p % bytes == 0 && pitch * e % bytes == 0;
}

}  // namespace st
