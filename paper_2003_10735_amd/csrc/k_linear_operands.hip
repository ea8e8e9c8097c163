// Operands of the dense layers' products that have to be made: copies of matrices whose addresses, strides or lengths the products' 16-byte
// loads do not take, and dz = dy act'(z) with the sums of its columns.
#include "st_linear.hpp"
#include "st_quantize.hpp"

#include <algorithm>

namespace st {

// ------------------------------------------------------------------------------------------------------ copies
// Eight values a thread along memory: 32 runs of 256 values a block, all of its loads under way at once.  `turn`: 64 x 64 through LDS, the other
// way round.
struct PackArgs { PackTask t[PACK_TASKS]; unsigned first[PACK_TASKS + 1], across[PACK_TASKS]; int count; };      // first block of each; blocks along a run
constexpr int PACK_RUNS = 32, PACK_VALUES = 256, TURN = 64;

template <class E> __device__ __forceinline__ void pack_block(const PackArgs& a, unsigned at_block, char* lds)
{
    int i = 0;
    while (i + 1 < a.count && at_block >= a.first[i + 1]) ++i;
    const PackTask& t = a.t[i];
    const unsigned block = at_block - a.first[i], down = block / a.across[i], along = block - down * a.across[i];
    const int ROWS = t.turn ? TURN : PACK_RUNS, VALUES = t.turn ? TURN : PACK_VALUES, LANES = VALUES / 8;
    const int64_t o0 = (int64_t)down * ROWS, i0 = (int64_t)along * VALUES;
    const int run = threadIdx.x % LANES, row = threadIdx.x / LANES, step = 256 / LANES;
    typedef E E8 __attribute__((ext_vector_type(8)));
    E* const to = (E*)t.to;
    constexpr int COUNT = PACK_RUNS * PACK_VALUES / 8 / 256;      // (turned: two of them)
    Raw8<E> v[COUNT];
    const int64_t at = i0 + run * 8;
#pragma unroll
    for (int h = 0; h < COUNT; ++h) {
        if (h * step >= ROWS) break;
        const E* x = (const E*)t.x + std::min(o0 + h * step + row, t.outer - 1) * t.pitch;
        if (t.inner < 8) v[h].load_short(x + at, at < t.inner ? (int)(t.inner - at) : 0);
        else v[h].load(x + run_start<8, int64_t>(at, t.inner));
    }
    const int64_t d = t.inner < 8 ? 0 : at - (t.inner - 8);
    E (*turned)[TURN + 16 / sizeof(E)] = (E(*)[TURN + 16 / sizeof(E)])lds;
#pragma unroll
    for (int h = 0; h < COUNT; ++h) {
        if (h * step >= ROWS) break;
        if (d > 0) v[h].down(d < 8 ? (int)d : 8);
        const int64_t o = o0 + h * step + row;
        E8 u;
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = from_f32<E>(v[h][e]);
        if (!t.turn) { if (o < t.outer && at < t.to_pitch) *(E8*)(to + o * t.to_pitch + at) = u; }      // (pitches are multiples of eight)
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) turned[run * 8 + e][h * step + row] = o < t.outer ? u[e] : from_f32<E>(0.f);
    }
    if (!t.turn) return;
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t i1 = i0 + h * 32 + row, o1 = o0 + run * 8;
        if (i1 >= t.inner || o1 >= t.to_pitch) continue;
        E8 u;
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = turned[h * 32 + row][run * 8 + e];
        *(E8*)(to + i1 * t.to_pitch + o1) = u;
    }
}

template <class E> __global__ __launch_bounds__(256) void k_linear_fill_zero(E* __restrict__ p, int64_t rows, int64_t cols, int64_t pitch)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) p[i / cols * pitch + i % cols] = from_f32<E>(0.f);
}
void linear_fill_zero(Ctx& c, void* p, int is_bf16, int64_t rows, int64_t cols, int64_t pitch)
{
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(rows * cols, 2048), 4096));
    if (is_bf16) ST_LAUNCH(c, "linear_fill_zero", k_linear_fill_zero<bf16>, grid, dim3(256), 0, (bf16*)p, rows, cols, pitch);
    else ST_LAUNCH(c, "linear_fill_zero", k_linear_fill_zero<float>, grid, dim3(256), 0, (float*)p, rows, cols, pitch);
}

// ------------------------------------------------------------------------------------------------------ dz
// A block takes 64 columns and a part of the rows, 32 rows at a time: eight threads a row, eight values each.  What lies column by column
// goes through LDS, 64 columns x 32 rows.  dz is rounded to the operands' type, or where a product asks for them to two bfloat16
// terms (2^-16 off at most, where one is 2^-8); the sums of its columns are of what it was before.  8192 tokens x 4096 channels: 43 us, 4.7 TB/s.
struct SlopeArgs { SlopeTask t; unsigned across, blocks; int rows_each; };

template <class T> __device__ __forceinline__ void load_rows(const GradSource& s, int64_t m0, int64_t m, int64_t n0, int64_t n, float (*turned)[33], float (&v)[8])
{
    const int run = threadIdx.x & 7, row = threadIdx.x >> 3;
    if (s.along) {
        const int64_t r = std::min(m0 + row, m - 1), at = n0 + run * 8;
        const T* x = (const T*)s.x + r * s.pitch;
        Raw8<T> u;
        if (n < 8) u.load_short(x + at, at < n ? (int)(n - at) : 0);
        else {
            u.load(x + run_start<8, int64_t>(at, n));
            const int64_t d = at - (n - 8);
            if (d > 0) u.down(d < 8 ? (int)d : 8);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u[e];
        return;
    }
    const int col = threadIdx.x >> 2, part = threadIdx.x & 3;      // 64 columns, eight rows of each a thread
    const int64_t c = std::min(n0 + col, n - 1), at = m0 + part * 8;
    const T* x = (const T*)s.x + c * s.pitch;
    Raw8<T> u;
    if (m < 8) u.load_short(x + at, at < m ? (int)(m - at) : 0);
    else {
        u.load(x + run_start<8, int64_t>(at, m));
        const int64_t d = at - (m - 8);
        if (d > 0) u.down(d < 8 ? (int)d : 8);
    }
    __syncthreads();      // (what was there has been read)
#pragma unroll
    for (int e = 0; e < 8; ++e) turned[col][part * 8 + e] = u[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = turned[run * 8 + e][row];
}

template <class E> __device__ __forceinline__ void store_dz(void* to, int64_t at, const float (&v)[8])
{
    typedef E E8 __attribute__((ext_vector_type(8)));
    E8 u;
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = from_f32<E>(v[e]);
    *(E8*)((E*)to + at) = u;
}

template <class T, class Z, int ACT> __device__ __forceinline__ void slope_rows(const SlopeArgs& a, unsigned block, float (*turned)[33], float (*sums)[64])
{
    const SlopeTask& t = a.t;
    const int64_t n0 = (int64_t)(block % a.across) * 64, part = block / a.across;
    const int64_t from = part * a.rows_each, to = std::min(from + a.rows_each, t.m);
    const int run = threadIdx.x & 7, row = threadIdx.x >> 3;
    float sum[8] = {};
    for (int64_t m0 = from; m0 < to; m0 += 32) {
        float v[8], z[8];
        load_rows<T>(t.dy, m0, t.m, n0, t.n, turned, v);
        if constexpr (ACT != ST_ACT_NONE) load_rows<Z>(t.pre, m0, t.m, n0, t.n, turned, z);
        if (m0 + row >= to) continue;      // (the last turn of the loop)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (ACT != ST_ACT_NONE) v[e] = slope_times<ACT>(v[e], z[e]);
            if (n0 + run * 8 + e >= t.n) v[e] = 0.f;
            sum[e] += v[e];
        }
        if (t.to && n0 + run * 8 < t.to_pitch) {
            const int64_t at = (m0 + row) * t.to_pitch + n0 + run * 8;
            if (t.to_bf16) store_dz<bf16>(t.to, at, v); else store_dz<float>(t.to, at, v);
            if (t.second) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float first = (float)(bf16)v[e];
                    v[e] = fabsf(first) < __builtin_inff() ? v[e] - first : 0.f;      // (an infinity is all in the first, a NaN in the first as well)
                }
                store_dz<bf16>(t.to, at + t.second, v);
            }
        }
    }
    if (!t.parts) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[row][run * 8 + e] = sum[e];
    __syncthreads();
    if (threadIdx.x < 64 && n0 + threadIdx.x < t.n) {
        float v = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) v += sums[r][threadIdx.x];
        t.parts[part * t.n + n0 + threadIdx.x] = v;
    }
}

template <class T, class Z> __device__ __forceinline__ void slope_block(const SlopeArgs& a, unsigned block, char* lds)
{
    float (*turned)[33] = (float(*)[33])lds, (*sums)[64] = (float(*)[64])(lds + 64 * 33 * 4);
    switch (a.t.act) {
    case ST_ACT_RELU: slope_rows<T, Z, ST_ACT_RELU>(a, block, turned, sums); break;
    case ST_ACT_GELU: slope_rows<T, Z, ST_ACT_GELU>(a, block, turned, sums); break;
    case ST_ACT_GELU_TANH: slope_rows<T, Z, ST_ACT_GELU_TANH>(a, block, turned, sums); break;
    case ST_ACT_SILU: slope_rows<T, Z, ST_ACT_SILU>(a, block, turned, sums); break;
    default: slope_rows<T, Z, ST_ACT_NONE>(a, block, turned, sums); break;
    }
}

// One launch makes all of a call's operands: dz first, whose blocks work longest, then the copies.
struct PrepareArgs { SlopeArgs slope; PackArgs pack; };
static_assert(sizeof(PrepareArgs) <= 4096, "kernel arguments");
template <class E> __global__ __launch_bounds__(256) void k_linear_prepare(const PrepareArgs a)
{
    __shared__ __align__(16) char lds[17408];
    static_assert(64 * 33 * 4 + 32 * 64 * 4 <= 17408 && 64 * (64 + 4) * 4 <= 17408, "room for either");
    if (blockIdx.x >= a.slope.blocks) { pack_block<E>(a.pack, blockIdx.x - a.slope.blocks, lds); return; }
    const SlopeTask& t = a.slope.t;
    if (t.dy.bf16) { if (t.pre.bf16) slope_block<bf16, bf16>(a.slope, blockIdx.x, lds); else slope_block<bf16, float>(a.slope, blockIdx.x, lds); }
    else { if (t.pre.bf16) slope_block<float, bf16>(a.slope, blockIdx.x, lds); else slope_block<float, float>(a.slope, blockIdx.x, lds); }
}

// Parts of the rows: about four blocks a compute unit, 32 rows at least; no more parts than the launch that adds them reads in passing (14400
// cells of 128 channels: 450 parts 6.4 us, 113 parts 9.5; 8192 tokens of 4096 channels in 16 parts 43 us, in 8 64, in 32 47).
static int slope_rows_each(int64_t m, int64_t n)
{
    const int64_t parts = std::min<int64_t>(512, std::max<int64_t>(1, 1024 / ceil_div(n, 64)));
    return (int)round_up(std::max<int64_t>(32, ceil_div(m, parts)), 32);
}
int linear_slope_parts(int64_t m, int64_t n) { return (int)ceil_div(m, slope_rows_each(m, n)); }

void linear_prepare(Ctx& c, const SlopeTask* slope, const PackTask* t, int count, int is_bf16)
{
    PrepareArgs a{};
    if (slope) {
        const unsigned across = (unsigned)ceil_div(slope->n, 64);
        a.slope = SlopeArgs{*slope, across, across * (unsigned)linear_slope_parts(slope->m, slope->n), slope_rows_each(slope->m, slope->n)};
    }
    for (int done = 0; done < count || a.slope.blocks;) {      // (a launch holds fewer than 2^32 threads)
        for (; done < count && (a.pack.count == 0 || a.pack.first[a.pack.count] < (1 << 22)); ++done) {
            const int i = a.pack.count++;
            a.pack.t[i] = t[done];
            a.pack.across[i] = (unsigned)ceil_div(t[done].inner, t[done].turn ? TURN : PACK_VALUES);
            a.pack.first[i + 1] = a.pack.first[i] + a.pack.across[i] * (unsigned)ceil_div(t[done].outer, t[done].turn ? TURN : PACK_RUNS);
        }
        const dim3 grid(a.slope.blocks + a.pack.first[a.pack.count]);
        if (is_bf16) ST_LAUNCH(c, "linear_prepare", k_linear_prepare<bf16>, grid, dim3(256), 0, a);
        else ST_LAUNCH(c, "linear_prepare", k_linear_prepare<float>, grid, dim3(256), 0, a);
        a = PrepareArgs{};
    }
}

}  // namespace st
