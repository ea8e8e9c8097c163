// Products of 8-bit integers on the matrix cores:  out = act((a b^T) * a_scale * b_scale + bias), both operands row by row along the
// contraction.
//
// v_mfma_i32_32x32x32_i8: D[32x32] += A[32x32] B[32x32].  Lane l supplies A[l % 32][16*(l/32) .. +15] and B[16*(l/32) .. +15][l % 32];
// it receives D[8*(r/4) + 4*(l/32) + r%4][l % 32] in register r.  The rows of b (output channels) are A's, so that four registers of a
// lane are four neighbouring channels of one token.
//
// A stage of 128 bytes of the contraction of a tile's rows goes from memory into LDS directly, 16 bytes a lane, eight rows a
// wavefront and instruction.  Chunk c (of 16 bytes) of row r lies in place c ^ (r / 2 % 8) of its row: two rows span the 64 banks, so lanes
// that read the same chunk of sixteen consecutive rows read sixteen different groups of four banks.  (With c ^ (r % 8) rows r and r + 8
// met: half of the LDS cycles were conflicts.)
#include "st_quantize.hpp"

#include <algorithm>

namespace st {

constexpr int BAND = 4;         // rows of tiles
constexpr int STAGE = 128;      // bytes of the contraction a stage holds

struct GemmArgs {
    Product p;
    FastDiv by_tiles, by_band;                // tiles of a split, tiles of a band of BAND rows of tiles
    int tiles_m;
    int splits, stages;                       // stages: of the whole contraction
    unsigned blocks;
};
struct GemmPair { GemmArgs g[2]; };

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

// One value's way out: scales, bias, ReLU.
struct Column { float scale, bias; };
__device__ __forceinline__ float finish(float sum, float a_scale, Column c, bool relu)
{
    const float v = sum * a_scale * c.scale + c.bias;
    return relu && v < 0.f ? 0.f : v;
}
__device__ __forceinline__ Column column_of(const Product& p, int64_t n)
{
    return n < p.n ? Column{p.b_scale[n], p.bias ? p.bias[n] : 0.f} : Column{0.f, 0.f};
}
// COUNT values of one row, channels n .. n + COUNT - 1: at once, or at the end of the row those that exist one by one.  (Stores that do not
// ask for room in L2 lose more than they give here: 8192 tokens 4096 -> 14336 444 us against 454, but 14400 tokens 256 -> 128 8.5 against 8.0,
// and odd pitches, whose lines are written in parts, 58.6 against 49.5 at 5480 tokens 532 -> 6367.)
template <int COUNT> __device__ __forceinline__ void store_out(const Product& p, int64_t m, int64_t n, const float (&v)[COUNT])
{
    if (p.out_bf16) {
        bf16* o = (bf16*)p.out + m * p.out_pitch + n;
        if (n + COUNT <= p.n) {
            typedef bf16 T __attribute__((ext_vector_type(COUNT)));
            typedef T T2 __attribute__((aligned(2)));
            T u;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) u[i] = (bf16)v[i];
            *(T2*)o = u;
            return;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) if (n + i < p.n) o[i] = (bf16)v[i];
    } else {
        float* o = (float*)p.out + m * p.out_pitch + n;
        if (n + COUNT <= p.n) {
            if constexpr (COUNT == 1) *o = v[0];
            else
#pragma unroll
                for (int i = 0; i < COUNT; i += 4) *(f32x4_4*)(o + i) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
            return;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) if (n + i < p.n) o[i] = v[i];
    }
}

// s_waitcnt vmcnt(N) alone; a barrier that memory accesses stay on their side of, without a wait of its own
#define ST_WAIT_VM(N) __builtin_amdgcn_s_waitcnt(((N) & 15) | (((N) >> 4) << 14) | 0x0F70)
#define ST_BARRIER()                    \
    do {                                \
        asm volatile("" ::: "memory");  \
        __builtin_amdgcn_s_barrier();   \
        asm volatile("" ::: "memory");  \
    } while (0)

// BM tokens x BN channels a block, WM x WN a wavefront, DEPTH stages under way.  No unit is full: a stage's loads, its LDS reads and its
// products overlap in part only, and a barrier a stage keeps the wavefronts together.  Us a launch, whole, with the loads alone and without
// the loop's loads; then shares of the busy compute units' clocks in which LDS is read (256 bytes each; 234 measured by reads alone) and
// the matrix cores work, and of the wavefronts' cycles that are waits:
//   256        8192 tokens 4096 -> 14336   443   363   385    26 %   58 %   30 %
//   128        4096 tokens 2048 -> 2048   23.7  17.4  21.4    40 %   46 %   44 %
//   128 deep   1536 tokens 4096 -> 1536   19.7  15.2  17.1    31 %   39 %   41 %
//   64         1024 tokens 2048 -> 1024    9.0   7.8   7.6    13 %   12 %   50 %
// The first is 2.2 POP/s at the 1.8 GHz that the products leave (the same product of zeros takes 15 % less).  A stage of the last is 0.23 us
// (1024 tokens 8192 -> 1024 20.4 us, half as long a sum 13.0), with 3 to 8 stages under way alike; its loads alone take 0.17, 95 bytes a ns.
template <int BM, int BN, int WM, int WN, int DEPTH>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_int8_product(const GemmPair pair)
{
    constexpr int WAVES = (BM / WM) * (BN / WN), AR = BN, BR = BM;     // A operand: channels, B operand: tokens
    constexpr int BUF = (AR + BR) * STAGE;
    extern __shared__ __align__(16) char lds[];
    const bool second = blockIdx.x >= pair.g[0].blocks;
    const GemmArgs& g = pair.g[second];
    const Product& p = g.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // An XCD gets a run of consecutive tiles, ordered in bands of four tiles of tokens: what its 32 compute units work on at a time is
    // 4 x 8 tiles, and a third less goes from memory to its L2 than with rows of tiles.
    const int block = xcd_band((int)blockIdx.x - (second ? (int)pair.g[0].blocks : 0), (int)g.blocks);
    const int split = __builtin_amdgcn_readfirstlane(fast_quot(block, g.by_tiles));
    const int tile = block - split * (int)g.by_tiles.d;
    const int band = __builtin_amdgcn_readfirstlane(fast_quot(tile, g.by_band)), in_band = tile - band * (int)g.by_band.d;
    const int high = min(BAND, g.tiles_m - band * BAND);
    const int tn = __builtin_amdgcn_readfirstlane(in_band / high), tm = band * BAND + in_band - tn * high;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int first = (int)((int64_t)g.stages * split / g.splits), last = (int)((int64_t)g.stages * (split + 1) / g.splits);

    // bytes readable from the tile's first row on: beyond them a load gives zeros
    const int64_t k16 = (p.k + 15) / 16 * 16, kq = (p.k + STAGE - 1) / STAGE * STAGE;
    const auto ra = operand(p.b + n0 * p.b_pitch, (p.n - n0 - 1) * p.b_pitch + k16);
    const auto rb = operand(p.a + m0 * p.a_pitch, (p.m - m0 - 1) * p.a_pitch + kq);
    static_assert(WAVES % 2 == 0, "a wavefront's eight rows begin at an even or at an odd multiple of eight in every load");
    const unsigned chunk = ((lane & 7) ^ ((lane >> 4) + 4 * (wave & 1))) * 16;
    const unsigned va = (unsigned)(wave * 8 + (lane >> 3)) * (unsigned)p.b_pitch + chunk;
    const unsigned vb = (unsigned)(wave * 8 + (lane >> 3)) * (unsigned)p.a_pitch + chunk;
    const unsigned sa = WAVES * 8 * (unsigned)p.b_pitch, sb = WAVES * 8 * (unsigned)p.a_pitch;
    auto stage = [&](int s, int buf) {
        char* to = lds + buf * BUF + wave * 8 * STAGE;
        unsigned oa = va + (unsigned)s * STAGE, ob = vb + (unsigned)s * STAGE;
#pragma unroll
        for (int i = 0; i < AR / 8 / WAVES; ++i, oa += sa) load_to_lds(ra, to + i * WAVES * 8 * STAGE, oa);
#pragma unroll
        for (int i = 0; i < BR / 8 / WAVES; ++i, ob += sb) load_to_lds(rb, to + (AR + i * WAVES * 8) * STAGE, ob);
    };

    constexpr int NA = WN / 32, NB = WM / 32, STEPS = STAGE / 32;
    const int wn = (wave % (BN / WN)) * WN, wm = (wave / (BN / WN)) * WM;
    const int r32 = lane & 31, half = lane >> 5;
    const int offA = (wn + r32) * STAGE, offB = (AR + wm + r32) * STAGE;
    i32x16 acc[NB][NA] = {};
    i32x4 a[2][NA], b[2][NB];
    auto fetch = [&](int buf, int ks, int to) {
        const char* L = lds + buf * BUF + ((ks * 2 + half) ^ (r32 >> 1 & 7)) * 16;
#pragma unroll
        for (int i = 0; i < NA; ++i) a[to][i] = *(const i32x4*)(L + offA + i * 32 * STAGE);
#pragma unroll
        for (int j = 0; j < NB; ++j) b[to][j] = *(const i32x4*)(L + offB + j * 32 * STAGE);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < NA; ++i) acc[j][i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[from][i], b[from][j], acc[j][i], 0, 0, 0);
    };
    // in the instruction stream: one LDS read, one matrix instruction, while there are reads
    auto interleave = [] {
#pragma unroll
        for (int i = 0; i < NA + NB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
    };
    // DEPTH stages are under way.  A stage's last step has its operands in registers when the barrier is passed, so what follows the
    // barrier is: the loads of the stage DEPTH later into the buffer that is done with, the next stage's first operands, the last step's
    // products.  (8192 tokens 4096 -> 14336 with the loads last: 432 us a call instead of 441 with operands that a cache holds, 460 instead of
    // 447 with others every call.)
    constexpr int LOADS = (AR + BR) / 8 / WAVES;      // of a wavefront and stage
    static_assert((DEPTH - 1) * LOADS < 64, "the counter of loads under way");
    // what the sums meet on their way out is asked for before the loop
    constexpr int PITCH = WN + 4, RUNS = WN / 8, ROWS = 64 / RUNS;
    const int run = lane % RUNS, row = lane / RUNS;
    const int64_t n = n0 + wn + run * 8;
    Column col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) col[i] = column_of(p, n + i);
    if (first < last) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) if (first + d < last) stage(first + d, d);
        if (first + DEPTH <= last) ST_WAIT_VM((DEPTH - 1) * LOADS); else ST_WAIT_VM(0);
        ST_BARRIER();
        fetch(0, 0, 0);
    }
    for (int s = first, buf = 0; s < last; ++s) {
#pragma unroll
        for (int ks = 0; ks < STEPS - 1; ++ks) {
            __builtin_amdgcn_sched_barrier(0);
            fetch(buf, ks + 1, (ks + 1) & 1);
            multiply(ks & 1);
            interleave();
        }
        __builtin_amdgcn_sched_barrier(0);
        // the next stage is there (behind it DEPTH - 2 may still be on their way), this one is read
        if (DEPTH > 2 && s + DEPTH <= last) ST_WAIT_VM((DEPTH - 2) * LOADS); else ST_WAIT_VM(0);
        __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0)
        ST_BARRIER();
        if (s + DEPTH < last) stage(s + DEPTH, buf);
        buf = buf + 1 == DEPTH ? 0 : buf + 1;
        if (s + 1 < last) fetch(buf, 0, 0);
        multiply((STEPS - 1) & 1);
    }

    // Out through LDS, 32 tokens of a wavefront at a time: sums go in four neighbouring channels at a time and come out as runs along a row.
    __syncthreads();
    static_assert(WAVES * 32 * PITCH * 4 <= DEPTH * BUF, "room for the sums");
    int* mine = (int*)lds + wave * 32 * PITCH;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        float sm[32 / ROWS];
#pragma unroll
        for (int h = 0; h < 32 / ROWS; ++h) sm[h] = p.a_scale[min(m0 + wm + j * 32 + h * ROWS + row, p.m - 1)];
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(i32x4*)(mine + r32 * PITCH + i * 32 + q * 8 + half * 4) =
                    i32x4{acc[j][i][q * 4], acc[j][i][q * 4 + 1], acc[j][i][q * 4 + 2], acc[j][i][q * 4 + 3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 32 / ROWS; ++h) {
            const int r = h * ROWS + row;
            const int64_t m = m0 + wm + j * 32 + r;
            const i32x4 lo = *(const i32x4*)(mine + r * PITCH + run * 8), hi = *(const i32x4*)(mine + r * PITCH + run * 8 + 4);
            if (m >= p.m) continue;
            if (g.splits > 1) {
                int* to = p.slabs + ((int64_t)split * p.m + m) * p.n + n;
                if (n + 8 <= p.n) { ((i32x4_4*)to)[0] = lo; ((i32x4_4*)to)[1] = hi; }
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (n + i < p.n) to[i] = i < 4 ? lo[i] : hi[i - 4];
                continue;
            }
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = finish((float)(i < 4 ? lo[i] : hi[i - 4]), sm[h], col[i], p.relu);
            store_out<8>(p, m, n, v);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// The slabs of split products, added in 64 bits, and what the product's own epilogue does otherwise.  3.5 us where there is little to add
// (a launch and two trips to memory), 14 for 2188 x 1185 in two parts.
__global__ __launch_bounds__(256) void k_int8_join(const GemmPair pair, int64_t first, int64_t all)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const bool second = i >= first;
        const GemmArgs& g = pair.g[second];
        const Product& p = g.p;
        const int64_t at = second ? i - first : i, size = p.m * p.n, m = at / p.n, n = at - m * p.n;
        int64_t sum = 0;
#pragma unroll 4
        for (int s = 0; s < g.splits; ++s) sum += p.slabs[(int64_t)s * size + at];
        const float v[1] = {finish((float)sum, p.a_scale[m], column_of(p, n), p.relu)};
        store_out<1>(p, m, n, v);
    }
}

// --------------------------------------------------------------------------------------------------- few tokens
// Up to 32 tokens: the weights are read once, by as many wavefronts as there are, and the tokens' codes many times.  A block takes 16
// channels, each of its eight wavefronts an eighth of the contraction, 16 bytes a lane straight from memory into
// v_mfma_i32_16x16x64_i8 (lane l supplies A[l % 16][16*(l/16) .. +15] and B[16*(l/16) .. +15][l % 16] and receives
// D[4*(l/16) + r][l % 16]); the eighths are added in LDS.  Latency bounds it: 1 token 2048 -> 5632 6.0 us (11.6 MB of weights, 1.9 TB/s),
// 12 tokens 4096 -> 4096 5.9 (17 MB, 2.9 TB/s).
//
// FUSED: every block quantises the tokens by itself, into LDS, while its first weights are on their way: the tokens are few, and a launch
// of its own for them takes longer than the product.
constexpr int FEW_WAVES = 8;

struct FewArgs {
    Product p;
    const void* x; int x_bf16; int64_t x_row, x_step;        // FUSED: the tokens as they are: elements between two, and between two values
    int per_wave;                                            // bytes of the contraction a wavefront takes, a multiple of 64
    int lds_pitch;                                           // FUSED: bytes between two tokens' codes in LDS
    int group, per_token;                                    // FUSED: wavefronts along a token, a power of two; a thread's runs of a token
};

template <class T> constexpr int few_keep() { return sizeof(T) == 2 ? 8 : 4; }      // runs of eight values in a thread's registers

// Threads go along a token, eight values each; where a token has fewer than 512 such runs, several tokens are taken at once.  A thread
// keeps all of its runs (KEEP at most) in registers between the search for the largest and the rounding.
template <class T>
__device__ __forceinline__ void few_quantize(const FewArgs& f, char* codes, unsigned* tops, float* scales)
{
    constexpr int KEEP = few_keep<T>();
    const Product& p = f.p;
    const int m = (int)p.m, k = (int)p.k, end = FEW_WAVES * f.per_wave;
    const int threads = f.group * 64, lane = threadIdx.x & (threads - 1);
    const int first = __builtin_amdgcn_readfirstlane(threadIdx.x / threads), step = FEW_WAVES / f.group;
    const bool whole = k >= 8 && f.x_step == 1;
    if ((int)threadIdx.x < m) tops[threadIdx.x] = 0;
    Raw8<T> v[KEEP];
    int r = first, c = 0;
#pragma unroll
    for (int j = 0; j < KEEP; ++j) {
        const int at = (c * threads + lane) * 8;
        if (r < m) {
            const T* row = (const T*)f.x + r * f.x_row;
            if (whole) v[j].load(row + run_start<8>(at, k)); else v[j].load_short(row + at * f.x_step, k - at, f.x_step);
        }
        if (++c == f.per_token) { c = 0; r += step; }
    }
    __syncthreads();
    r = first; c = 0;
#pragma unroll
    for (int j = 0; j < KEEP; ++j) {
        if (r < m) {
            const int d = (c * threads + lane) * 8 - (k - 8);
            if (whole && d > 0) v[j].down(min(d, 8));
            unsigned top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[j][i]));
            top = wave_max(top);
            if ((threadIdx.x & 63) == 0) atomicMax(&tops[r], top);
        }
        if (++c == f.per_token) { c = 0; r += step; }
    }
    __syncthreads();
    r = first; c = 0;
#pragma unroll
    for (int j = 0; j < KEEP; ++j) {
        if (r < m) {
            float s;
            v[j].repack();
            const float mult = row_multiplier(tops[r], &s);
            if (c == 0 && lane == 0) scales[r] = s;
            const int at = (c * threads + lane) * 8;
            if (at < end)
                *(uint2*)(codes + r * f.lds_pitch + at) =
                    make_uint2(pack4(code_of(v[j][0], mult), code_of(v[j][1], mult), code_of(v[j][2], mult), code_of(v[j][3], mult)),
                               pack4(code_of(v[j][4], mult), code_of(v[j][5], mult), code_of(v[j][6], mult), code_of(v[j][7], mult)));
        }
        if (++c == f.per_token) { c = 0; r += step; }
    }
}

template <int NT, bool FUSED>
__global__ __launch_bounds__(FEW_WAVES * 64, 4) void k_int8_few(const FewArgs f)
{
    constexpr int AHEAD = FUSED ? 8 : 4;             // 64 bytes of the contraction each: loads under way twice over
    extern __shared__ __align__(16) char lds[];      // the wavefronts' sums [8][NT * 256]; FUSED: the codes behind them
    __shared__ unsigned tops[NT * 16];
    __shared__ float scales[NT * 16];
    const Product& p = f.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* codes = lds + FEW_WAVES * NT * 1024;
    const auto rb = operand(p.a, FUSED ? 0 : p.m * p.a_pitch);
    const unsigned kq = (unsigned)((p.k + 63) / 64 * 64);
    const unsigned from = (unsigned)wave * f.per_wave, to = from + f.per_wave < kq ? from + f.per_wave : kq;
    const unsigned va = (lane & 15) * (unsigned)p.b_pitch + (lane >> 4) * 16;
    struct Group { i32x4 a[AHEAD], b[FUSED ? 1 : NT][FUSED ? 1 : AHEAD]; };
    unsigned vb[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {      // (columns beyond the tokens are not used)
        const unsigned token = min(t * 16 + (lane & 15), (int)p.m - 1);
        vb[t] = token * (unsigned)(FUSED ? f.lds_pitch : p.a_pitch) + (lane >> 4) * 16;
    }
    auto channels = [&](int64_t n0) {
        const int64_t rows = p.n - n0 < 16 ? p.n - n0 : 16;
        return operand(p.b + n0 * p.b_pitch, (rows - 1) * p.b_pitch + (p.k + 15) / 16 * 16);
    };
    auto ask = [&](__amdgpu_buffer_rsrc_t ra, unsigned k, Group& w) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {      // (an offset beyond the buffer: zeros, and nothing is read)
            const bool there = k + u * 64 < to;
            w.a[u] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, (int)(there ? va + k + u * 64 : 0xfffffff0u), 0, 0));
            if constexpr (!FUSED)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    w.b[t][u] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rb, (int)(there ? vb[t] + k + u * 64 : 0xfffffff0u), 0, 0));
        }
    };
    int64_t n0 = (int64_t)blockIdx.x * 16;
    auto ra = channels(n0);
    Group g[2];
    ask(ra, from, g[0]);
    Column col = column_of(p, n0 + (threadIdx.x & 15));
    if constexpr (FUSED) {
        if (f.x_bf16) few_quantize<bf16>(f, codes, tops, scales); else few_quantize<float>(f, codes, tops, scales);
        __syncthreads();
    }
    i32x4 acc[NT];
    auto use = [&](unsigned k, const Group& w) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if constexpr (FUSED) {
                if (k + u * 64 >= to) break;
                acc[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w.a[u], *(const i32x4*)(codes + vb[0] + k + u * 64), acc[0], 0, 0, 0);
            } else
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w.a[u], w.b[t][u], acc[t], 0, 0, 0);
        }
    };
    while (true) {
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = i32x4{0, 0, 0, 0};
        for (unsigned k = from; k < to; k += 2 * AHEAD * 64) {
            if (k + AHEAD * 64 < to) ask(ra, k + AHEAD * 64, g[1]);
            use(k, g[0]);
            if (k + AHEAD * 64 >= to) break;
            if (k + 2 * AHEAD * 64 < to) ask(ra, k + 2 * AHEAD * 64, g[0]);
            use(k + AHEAD * 64, g[1]);
        }
        const int64_t at = n0, next = FUSED ? n0 + (int64_t)gridDim.x * 16 : p.n;
        const Column mine = col;
        if (next < p.n) {      // the next channels' weights, while these are added
            ra = channels(next);
            ask(ra, from, g[0]);
            col = column_of(p, next + (threadIdx.x & 15));
        }
        int* part = (int*)lds;
#pragma unroll
        for (int t = 0; t < NT; ++t) *(i32x4*)(part + (wave * NT + t) * 256 + (lane & 15) * 16 + (lane >> 4) * 4) = acc[t];
        __syncthreads();
        for (int i = threadIdx.x; i < NT * 256; i += FEW_WAVES * 64) {
            const int64_t m = i >> 4, n = at + (i & 15);
            if (m >= p.m || n >= p.n) continue;
            int sum = 0;
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) sum += part[w * NT * 256 + i];
            const float v[1] = {finish((float)sum, FUSED ? scales[m] : p.a_scale[m], mine, p.relu)};
            store_out<1>(p, m, n, v);
        }
        if (next >= p.n) break;
        n0 = next;
        __syncthreads();
    }
}

static int64_t few_per_wave(int64_t k) { return round_up(ceil_div(k, FEW_WAVES), 64); }
static int64_t few_lds(int64_t m, int64_t k) { return m * (FEW_WAVES * few_per_wave(k) + 16); }
// wavefronts along a token, and runs of eight values that a thread has of one
static void few_shape(int64_t m, int64_t k, int* group, int* per_token)
{
    *group = FEW_WAVES;
    while (*group > 1 && (*group / 2) * 512 >= FEW_WAVES * few_per_wave(k) && FEW_WAVES / *group < m) *group /= 2;
    *per_token = (int)ceil_div(FEW_WAVES * few_per_wave(k), *group * 512);
}
// FUSED where the tokens are those of one matrix-core tile and a thread's share of them fits its registers.  From five tokens on the
// tiled product with a quantising launch before it streams large weights faster (us a call: 8 tokens 4096 -> 4096 9.5 and 14.1, 4096 -> 14336
// 18.7 and 15.6; 4 tokens 4096 -> 14336 16.0 and 15.5, one token 12.8 and 15.3).
bool few_fused(int64_t m, int64_t n, int64_t k, int is_bf16)
{
    if (m > 16 || (m > 4 && n * k > 40000000)) return false;
    int group, per_token;
    few_shape(m, k, &group, &per_token);
    return ceil_div(m, FEW_WAVES / group) * per_token <= (is_bf16 ? few_keep<bf16>() : few_keep<float>());
}
// Otherwise, behind a quantising launch, against the tiled product: 12 tokens 4096 -> 4096 10.2 and 14.1, 32 tokens 11.6 and 14.3, 17 tokens
// 4096 -> 1024 10.4 and 14.2; but 16 tokens 4096 -> 14336 22.6 and 15.6, 32 tokens 8192 -> 500 16.4 and 14.2, 64 tokens 4096 -> 4096 15.8 and 14.5.
bool few_tokens(int64_t m, int64_t n, int64_t k) { return m <= 32 && n <= 8192 && k <= 4096; }

template <int NT, bool FUSED> static void few_launch(Ctx& c, const FewArgs& f)
{
    const size_t sums = (size_t)FEW_WAVES * NT * 1024, lds = sums + (FUSED ? (size_t)few_lds(f.p.m, f.p.k) : 0);
    ensure_dynamic_lds((const void*)k_int8_few<NT, FUSED>, FUSED ? 80 * 1024 : lds);
    // FUSED: two blocks a compute unit, every one with as many groups of channels as the others or one less
    const int64_t groups = ceil_div(f.p.n, 16), each = FUSED ? ceil_div(groups, 512) : 1;
    ST_LAUNCH(c, "int8_few", (k_int8_few<NT, FUSED>), dim3((unsigned)ceil_div(groups, each)), dim3(FEW_WAVES * 64), lds, f);
}
void product_few(Ctx& c, const Product& p, const QuantSource* x)
{
    FewArgs f{p, nullptr, 0, 0, 0, (int)few_per_wave(p.k), (int)(FEW_WAVES * few_per_wave(p.k) + 16), 0, 0};
    if (x) {
        f.x = x->x; f.x_bf16 = x->bf16; f.x_row = x->along ? x->pitch : 1; f.x_step = x->along ? 1 : x->pitch;
        few_shape(p.m, p.k, &f.group, &f.per_token);
        few_launch<1, true>(c, f);
    } else if (p.m <= 16) few_launch<1, false>(c, f);
    else few_launch<2, false>(c, f);
}

// ------------------------------------------------------------------------------------------------- narrow layers
// Many tokens through a small layer (the cells of a feature map): a block takes 32 tokens, quantises them into LDS and multiplies them by
// all of the weights, 32 channels a wavefront and v_mfma_i32_32x32x32_i8 at a time, which come from a cache.  The tokens are read once, no
// codes go through memory and one launch does it all.  Eight threads take a token, eight values at a time; RUNS of them cover a token.
// 14400 tokens 256 -> 128: 7.6 us, 1.5 TB/s, in 450 blocks that each read, quantise, multiply and store once, so their latencies add up.
struct NarrowArgs { Product p; const void* x; int64_t x_pitch; };
constexpr int NARROW_TOKENS = 32;

template <class T, int RUNS> __global__ __launch_bounds__(256) void k_int8_narrow(const NarrowArgs f)
{
    constexpr int STEPS = RUNS * 2, PITCH = RUNS * 64 + 16, OUT = 128 + 4;       // codes: 16 bytes on, so that rows begin on other banks
    __shared__ __align__(16) char codes[NARROW_TOKENS * PITCH];
    __shared__ __align__(16) int sums[NARROW_TOKENS * OUT];
    __shared__ float scales[NARROW_TOKENS];
    const Product& p = f.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)blockIdx.x * NARROW_TOKENS;
    const int k = (int)p.k, n = (int)p.n;
    const int r32 = lane & 31, half = lane >> 5;
    i32x4 w[STEPS];
    auto weights = [&](int n0) {
        const int rows = min(32, n - n0);
        if (rows <= 0) return;
        const auto rsrc = operand(p.b + n0 * p.b_pitch, (rows - 1) * p.b_pitch + (k + 15) / 16 * 16);
        const unsigned at = r32 * (unsigned)p.b_pitch + half * 16;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            w[s] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(s * 32 < k ? at + s * 32 : 0xfffffff0u), 0, 0));
    };

    const int token = threadIdx.x >> 3, t8 = threadIdx.x & 7;
    const bool there = m0 + token < p.m;
    const T* x = (const T*)f.x + (there ? m0 + token : 0) * f.x_pitch;
    Raw8<T> v[RUNS];
    load_row<true>(x, k, [&](int i) { return (i * 8 + t8) * 8; }, v);
    weights(wave * 32);
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, abs_bits(v[i][e]));
#define ST_DPP(CTRL) top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, CTRL, 0xf, 0xf, false))
    ST_DPP(0xb1); ST_DPP(0x4e); ST_DPP(0x141);      // lanes 1 and 2 across in fours, then the eight's other four
#undef ST_DPP
    float scale;
    const float mult = row_multiplier(top, &scale);
    if (t8 == 0) scales[token] = scale;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        v[i].repack();
        *(uint2*)(codes + token * PITCH + (i * 8 + t8) * 8) =
            make_uint2(pack4(code_of(v[i][0], mult), code_of(v[i][1], mult), code_of(v[i][2], mult), code_of(v[i][3], mult)),
                       pack4(code_of(v[i][4], mult), code_of(v[i][5], mult), code_of(v[i][6], mult), code_of(v[i][7], mult)));
    }
    __syncthreads();
    const int run = threadIdx.x & 15, row = threadIdx.x >> 4;
    for (int base = 0; base < n; base += 128) {
        const int c = base + run * 8;
        Column col[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) col[i] = column_of(p, c + i);
        if (base + wave * 32 < n) {
            i32x16 acc = {};
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
                if (s * 32 < k) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[s], *(const i32x4*)(codes + r32 * PITCH + s * 32 + half * 16), acc, 0, 0, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(i32x4*)(sums + r32 * OUT + wave * 32 + q * 8 + half * 4) = i32x4{acc[q * 4], acc[q * 4 + 1], acc[q * 4 + 2], acc[q * 4 + 3]};
        }
        if (base + 128 < n) weights(base + 128 + wave * 32);
        __syncthreads();
        if (c < n) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = h * 16 + row;
                if (m0 + r >= p.m) break;
                const i32x4 lo = *(const i32x4*)(sums + r * OUT + run * 8), hi = *(const i32x4*)(sums + r * OUT + run * 8 + 4);
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = finish((float)(i < 4 ? lo[i] : hi[i - 4]), scales[r], col[i], p.relu);
                store_out<8>(p, m0 + r, c, o);
            }
        }
        if (base + 128 < n) __syncthreads();
    }
}

// Every block reads all of the weights: up to 64 KB of them.  Against a quantising launch and the tiled product, us a call: 14400 tokens
// 256 -> 128 6.7 and 11.6, 256 -> 256 10.8 and 13.3, 512 -> 128 9.6 and 15.0, 200000 tokens 256 -> 128 57.5 and 91.7; but 1000 tokens 512 -> 256
// 11.1 and 9.2, 60000 tokens 512 -> 256 56 and 41.
bool narrow_layer(int64_t m, int64_t n, int64_t k)
{
    return m > 32 && k <= 512 && n <= 256 && k * n <= 65536;
}
template <class T> static void narrow_launch(Ctx& c, const NarrowArgs& f)
{
    const dim3 grid((unsigned)ceil_div(f.p.m, NARROW_TOKENS));
    if (f.p.k <= 128) ST_LAUNCH(c, "int8_narrow", (k_int8_narrow<T, 2>), grid, dim3(256), 0, f);
    else if (f.p.k <= 256) ST_LAUNCH(c, "int8_narrow", (k_int8_narrow<T, 4>), grid, dim3(256), 0, f);
    else ST_LAUNCH(c, "int8_narrow", (k_int8_narrow<T, 8>), grid, dim3(256), 0, f);
}
void product_narrow(Ctx& c, const Product& p, const QuantSource& x)
{
    const NarrowArgs f{p, x.x, x.pitch};
    if (x.bf16) narrow_launch<bf16>(c, f); else narrow_launch<float>(c, f);
}

// --------------------------------------------------------------------------------------- choice of tile and split
static int64_t tiles_of(const Extent& e, int tile) { return ceil_div(e.m, tile) * ceil_div(e.n, tile); }
Form form_of(const Extent* e, int count)
{
    auto total = [&](int tile) { int64_t t = 0; for (int i = 0; i < count; ++i) t += tiles_of(e[i], tile); return t; };
    auto stages_of = [&](int tile) { int64_t w = 0; for (int i = 0; i < count; ++i) w += tiles_of(e[i], tile) * ceil_div(e[i].k, STAGE); return w; };
    Form f = {64, {1, 1}};
    // (a tile of five stages or fewer is begun and ended most of its time: smaller ones, two a compute unit, overlap; 5480 tokens 532 -> 6367
    // 48.5 us against 62, 14400 tokens 256 -> 2048 33.0 against 36.4; but 8192 tokens 1024 -> 8192 107 against 96)
    if (total(256) >= 192 && stages_of(256) > 5 * total(256)) f.tile = 256;
    // (small tiles fill the card with two a compute unit: 1536 tokens 4096 -> 1536, 576 of them, 33.9 us, with large ones 27.1; 1500 tokens
    // 2048 -> 1700, 648, 21.7 and 18.7; but 512 tokens 4096 -> 4096, 512, 23.1 and 33.6, 2000 tokens 1000 -> 1000, 512, 11.7 and 12.7)
    else if (total(64) > 512) f.tile = 128;
    // every block about the same number of stages, 256 blocks, eight stages each at least; up to 16 stages the parts' join costs more than
    // it gives (333 tokens 1000 -> 1003: 11.8 us, in two parts 15.6; 65 tokens 8192 -> 128 in eight parts: 12.7, in four 15.0)
    const int64_t each = std::max<int64_t>(8, ceil_div(stages_of(f.tile), 256));
    for (int i = 0; i < count; ++i) {
        const int64_t stages = ceil_div(e[i].k, STAGE);
        int64_t s = stages > 16 ? stages / each : 1;
        // (beside another product, blocks that would go on for 20 stages when the others are done: over 26 backward passes that this changes,
        // 24 of them drawn at random, 0.83 to 1.05 of the time without, 0.90 on average; 13282 tokens 442 -> 2258 112 us instead of 134; 1500
        // tokens 8192 -> 1700, alone, 53.6 instead of 42.6, so there not)
        if (count > 1 && f.tile == 128 && s == 1 && stages >= each + 20) s = 2;
        s = std::max(s, ceil_div(stages, ST_INT8_MAX_SUM / STAGE));    // what int32 can hold
        f.splits[i] = (int)std::max<int64_t>(s, 1);
    }
    return f;
}

template <int BM, int BN, int WM, int WN, int DEPTH>
static void launch(Ctx& c, const GemmPair& g)
{
    constexpr size_t lds = (size_t)DEPTH * (BM + BN) * STAGE;
    ensure_dynamic_lds((const void*)k_int8_product<BM, BN, WM, WN, DEPTH>, lds);
    constexpr const char* name = BM == 256 ? "int8_product_256" : BM == 64 ? "int8_product_64" : DEPTH > 2 ? "int8_product_128_deep" : "int8_product_128";
    ST_LAUNCH(c, name, (k_int8_product<BM, BN, WM, WN, DEPTH>), dim3(g.g[0].blocks + g.g[1].blocks), dim3((BM / WM) * (BN / WN) * 64), lds, g);
}

void products(Ctx& c, const Product* p, int count)
{
    if (count == 0) return;
    Extent e[2];
    for (int i = 0; i < count; ++i) e[i] = {p[i].m, p[i].n, p[i].k};
    const Form f = form_of(e, count);
    GemmPair g{}, joined{};
    int n_joined = 0;
    int64_t cells[2] = {0, 0};
    for (int i = 0; i < count; ++i) {
        const int64_t tm = ceil_div(p[i].m, f.tile), tn = ceil_div(p[i].n, f.tile);
        g.g[i] = GemmArgs{p[i], fast_div((int)(tm * tn)), fast_div((int)(tn * BAND)), (int)tm, f.splits[i],
                          (int)ceil_div(p[i].k, STAGE), (unsigned)(tm * tn * f.splits[i])};
        if (f.splits[i] > 1) { cells[n_joined] = p[i].m * p[i].n; joined.g[n_joined++] = g.g[i]; }
    }
    if (f.tile == 256) launch<256, 256, 128, 64, 2>(c, g);
    // (one block a compute unit: deeper; 1000 tokens 4000 -> 4000 31.0 us against 34.8; else two blocks: 4096 tokens 2048 -> 2048 32.1 against 40.4)
    else if (f.tile == 128 && g.g[0].blocks + g.g[1].blocks <= 256) launch<128, 128, 64, 32, 4>(c, g);
    else if (f.tile == 128) launch<128, 128, 64, 32, 2>(c, g);
    else launch<64, 64, 32, 32, 4>(c, g);
    if (n_joined) {
        const int64_t all = cells[0] + cells[1], blocks = ceil_div(all, 256);
        ST_LAUNCH(c, "int8_join", k_int8_join, dim3((unsigned)(blocks > 8192 ? 8192 : blocks)), dim3(256), 0, joined, cells[0], all);
    }
}

}  // namespace st
