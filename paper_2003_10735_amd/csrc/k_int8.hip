// Products of 8-bit integers on the matrix cores:  out = act((a b^T) * a_scale * b_scale + bias), both operands row by row along the
// contraction.
//
// v_mfma_i32_32x32x32_i8: D[32x32] += A[32x32] B[32x32].  Lane l supplies A[l % 32][16*(l/32) .. +15] and B[16*(l/32) .. +15][l % 32];
// it receives D[8*(r/4) + 4*(l/32) + r%4][l % 32] in register r.  The rows of b (output channels) are A's, so that four registers of a
// lane are four neighbouring channels of one token.
//
// A stage of 128 bytes of the contraction of a tile's rows goes from memory into LDS directly, 16 bytes a lane, eight rows a
// wavefront and instruction.  Chunk c (of 16 bytes) of row r lies in place c ^ (r & 7) of its row: lanes that read the same chunk of
// eight consecutive rows then read eight different groups of banks.
#include "st_dense.hpp"

namespace st {

constexpr int STAGE = 128;      // bytes of the contraction a stage holds

struct GemmArgs {
    Product p;
    int tiles_m, tiles_n, splits, stages;     // stages: of the whole contraction
    int* slabs;                               // [splits, m, n] where splits > 1
};

// 16 bytes a lane from `rsrc` + voff to LDS at `lds` + 16 * lane (the whole offset is the lanes': a scalar one takes no part in the
// comparison with the buffer's size)
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t rsrc, char* lds, unsigned voff)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, (int)voff, 0, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t operand(const int8_t* base, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)(unsigned)(bytes < 0xffffffffll ? bytes : 0xffffffffll), 0x00020000);
}

// BM tokens x BN channels a block, WM x WN a wavefront.
template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_int8_product(const GemmArgs g)
{
    constexpr int WAVES = (BM / WM) * (BN / WN), AR = BN, BR = BM;     // A operand: channels, B operand: tokens
    constexpr int BUF = (AR + BR) * STAGE;
    extern __shared__ __align__(16) char lds[];
    const Product& p = g.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile = blockIdx.x;
    const int tiles = g.tiles_m * g.tiles_n, split = tile / tiles;
    tile -= split * tiles;
    const int tm = tile / g.tiles_n, tn = tile - tm * g.tiles_n;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int first = (int)((int64_t)g.stages * split / g.splits), last = (int)((int64_t)g.stages * (split + 1) / g.splits);

    // bytes readable from the tile's first row on: beyond them a load gives zeros
    const int64_t k16 = (p.k + 15) / 16 * 16, kq = (p.k + STAGE - 1) / STAGE * STAGE;
    const auto ra = operand(p.b + n0 * p.b_pitch, (p.n - n0 - 1) * p.b_pitch + k16);
    const auto rb = operand(p.a + m0 * p.a_pitch, (p.m - m0 - 1) * p.a_pitch + kq);
    const unsigned chunk = ((lane & 7) ^ (lane >> 3)) * 16;
    const unsigned va = (unsigned)(lane >> 3) * (unsigned)p.b_pitch + chunk, vb = (unsigned)(lane >> 3) * (unsigned)p.a_pitch + chunk;
    auto stage = [&](int s, int buf) {
        char* to = lds + buf * BUF;
#pragma unroll
        for (int i = 0; i < AR / 8 / WAVES; ++i) {
            const int r = (i * WAVES + wave) * 8;
            load_to_lds(ra, to + r * STAGE, va + (unsigned)r * (unsigned)p.b_pitch + (unsigned)s * STAGE);
        }
#pragma unroll
        for (int i = 0; i < BR / 8 / WAVES; ++i) {
            const int r = (i * WAVES + wave) * 8;
            load_to_lds(rb, to + (AR + r) * STAGE, vb + (unsigned)r * (unsigned)p.a_pitch + (unsigned)s * STAGE);
        }
    };

    constexpr int NA = WN / 32, NB = WM / 32;
    const int wn = (wave % (BN / WN)) * WN, wm = (wave / (BN / WN)) * WM;
    const int r32 = lane & 31, half = lane >> 5;
    i32x16 acc[NB][NA] = {};
    if (first < last) stage(first, 0);
    for (int s = first; s < last; ++s) {
        const int buf = (s - first) & 1;
        __builtin_amdgcn_s_waitcnt(0x0f70);    // vmcnt(0): this stage has arrived
        __syncthreads();                       // .. for every wavefront, and every one is done with the other buffer
        if (s + 1 < last) stage(s + 1, buf ^ 1);
        const char* A = lds + buf * BUF + (wn + r32) * STAGE;
        const char* B = lds + buf * BUF + (AR + wm + r32) * STAGE;
#pragma unroll
        for (int ks = 0; ks < STAGE / 32; ++ks) {
            const int place = ((ks * 2 + half) ^ (r32 & 7)) * 16;
            i32x4 a[NA], b[NB];
#pragma unroll
            for (int i = 0; i < NA; ++i) a[i] = *(const i32x4*)(A + i * 32 * STAGE + place);
#pragma unroll
            for (int j = 0; j < NB; ++j) b[j] = *(const i32x4*)(B + j * 32 * STAGE + place);
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < NA; ++i) acc[j][i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[j][i], 0, 0, 0);
        }
    }

#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int64_t m = m0 + wm + j * 32 + r32;
        if (m >= p.m) continue;
        if (g.splits > 1) {
            int* to = g.slabs + ((int64_t)split * p.m + m) * p.n;
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t n = n0 + wn + i * 32 + 8 * (r / 4) + 4 * half + r % 4;
                    if (n < p.n) to[n] = acc[j][i][r];
                }
            continue;
        }
        const float sm = p.a_scale[m];
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t n = n0 + wn + i * 32 + 8 * (r / 4) + 4 * half + r % 4;
                if (n >= p.n) continue;
                float v = (float)acc[j][i][r] * sm * p.b_scale[n];
                if (p.bias) v += p.bias[n];
                if (p.relu) v = v < 0.f ? 0.f : v;
                if (p.out_bf16) ((bf16*)p.out)[m * p.out_pitch + n] = (bf16)v;
                else ((float*)p.out)[m * p.out_pitch + n] = v;
            }
    }
}

// The slabs of a split product, added in 64 bits, and what the product's own epilogue does otherwise.
__global__ __launch_bounds__(256) void k_int8_join(const GemmArgs g)
{
    const Product& p = g.p;
    const int64_t all = p.m * p.n;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t m = at / p.n, n = at - m * p.n;
        int64_t sum = 0;
        for (int s = 0; s < g.splits; ++s) sum += g.slabs[(int64_t)s * all + at];
        float v = (float)sum * p.a_scale[m] * p.b_scale[n];
        if (p.bias) v += p.bias[n];
        if (p.relu) v = v < 0.f ? 0.f : v;
        if (p.out_bf16) ((bf16*)p.out)[m * p.out_pitch + n] = (bf16)v;
        else ((float*)p.out)[m * p.out_pitch + n] = v;
    }
}

// --------------------------------------------------------------------------------------- choice of tile and split
struct Form { int bm, bn, splits; };
static Form form_of(int64_t m, int64_t n, int64_t k)
{
    const int64_t stages = ceil_div(k, STAGE);
    Form f = {64, 64, 1};
    if (ceil_div(m, 256) * ceil_div(n, 256) >= 192) f = {256, 256, 1};
    else if (ceil_div(m, 128) * ceil_div(n, 128) >= 192) f = {128, 128, 1};
    const int64_t tiles = ceil_div(m, f.bm) * ceil_div(n, f.bn);
    int64_t s = 512 / tiles;                                   // two blocks a compute unit
    if (s > stages / 4) s = stages / 4;                        // four stages each at least
    if (s < 1) s = 1;
    const int64_t least = ceil_div(stages, ST_INT8_MAX_SUM / STAGE);    // what int32 can hold
    if (s < least) s = least;
    f.splits = (int)s;
    return f;
}

size_t product_slab_bytes(int64_t m, int64_t n, int64_t k)
{
    const Form f = form_of(m, n, k);
    return f.splits > 1 ? (size_t)f.splits * m * n * 4 : 0;
}

template <int BM, int BN, int WM, int WN>
static void launch(Ctx& c, const GemmArgs& g)
{
    constexpr size_t lds = 2 * (BM + BN) * STAGE;
    ensure_dynamic_lds((const void*)k_int8_product<BM, BN, WM, WN>, lds);
    ST_LAUNCH(c, "int8_product", (k_int8_product<BM, BN, WM, WN>), dim3((unsigned)g.tiles_m * g.tiles_n * g.splits),
              dim3((BM / WM) * (BN / WN) * 64), lds, g);
}

void product(Ctx& c, const Product& p, int* slabs)
{
    const Form f = form_of(p.m, p.n, p.k);
    GemmArgs g{p, (int)ceil_div(p.m, f.bm), (int)ceil_div(p.n, f.bn), f.splits, (int)ceil_div(p.k, STAGE), slabs};
    if (f.bm == 256) launch<256, 256, 128, 64>(c, g);
    else if (f.bm == 128) launch<128, 128, 64, 64>(c, g);
    else launch<64, 64, 32, 32>(c, g);
    if (f.splits > 1) {
        const int64_t blocks = ceil_div(p.m * p.n, 256);
        ST_LAUNCH(c, "int8_join", k_int8_join, dim3((unsigned)(blocks > 8192 ? 8192 : blocks)), dim3(256), 0, g);
    }
}

}  // namespace st
