// Products of bfloat16 or float32 operands on the matrix cores, with bias, activation and residual on their way out:
//   out = act(a b^T + bias) + residual
//
// Either operand lies row by row along the contraction, or across it (a dense layer's gradients contract over what their operands' rows
// are); no operand is copied to be turned.  A stage of 128 bytes of the contraction of a row (64 values, or 32 of float32) goes from
// memory into LDS directly, 16 bytes a lane, and from there into fragments of 16 bytes a lane:
//   v_mfma_f32_32x32x16_bf16: lane l supplies A[l % 32][8*(l/32) .. +7] and B[8*(l/32) .. +7][l % 32];
//   v_mfma_f32_32x32x2_f32:   lane l supplies A[l % 32][l/32] and B[l/32][l % 32]: of the 16 bytes one value an instruction, so that an
//                             instruction's two positions of the contraction lie four apart, for both operands alike;
// both give D[8*(r/4) + 4*(l/32) + r%4][l % 32] in register r.  The rows of b (output channels) are A's, so that four registers of a lane
// are four neighbouring channels of one token.
//
// Along: a row takes 128 bytes of LDS; chunk c (of 16 bytes) of row r lies in place c ^ (r / 2 % 8), so that lanes that read the same
// chunk of sixteen consecutive rows read sixteen different groups of four banks.
// Across: a position k of the contraction takes the tile's rows, R values next to each other.  bfloat16: ds_read_b64_tr_b16 turns 4 x 16
// values in a group of sixteen lanes: lane j gives the address of four rows' values, 4*(j%4) .., of position j/4, and gets the four positions'
// values of row j.  The 64 bytes that a position gives are moved by k % 4 times 64 bytes (R = 64: by 64 bytes where k / 2 is odd; R = 32: not), so
// that four positions of 32 rows meet no bank twice.  float32: 32 lanes read 32 rows' values at one position, the two halves of a wavefront four
// positions apart, moved by 128 bytes.
#include "st_linear.hpp"
#include "st_quantize.hpp"

#include <algorithm>

namespace st {

constexpr int BAND = 4;         // rows of tiles
constexpr int STAGE = 128;      // bytes of the contraction a stage holds
constexpr unsigned OUTSIDE = 0xffffff00u;      // an offset behind every buffer: a load gives zeros

struct GemmArgs {
    LinearProduct p;
    FastDiv by_tiles, by_band;                // tiles of a split, tiles of a band of BAND rows of tiles
    int tiles_m;
    int splits, stages, once;                 // stages: of the whole contraction, once: of one of its terms
    unsigned blocks;
};
struct GemmPair { GemmArgs g[2]; ColumnSums sums; };

typedef short s16x4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane from `rsrc` + voff to LDS at `lds` + 16 * lane (the whole offset is the lanes': a scalar one takes no part in the
// comparison with the buffer's size).  Written out, because the compiler has every transposing LDS read wait for all loads of its own
// builtin that are under way, whatever they write (8192 tokens 4096 -> 4096, dz^T x: 256 us that way); the waits that are needed stand
// where the stages change.  No register is written; M0, which holds the place in LDS, is an operand, so that the compiler sets it and knows what it
// holds.  The pause covers M0 and a scalar register that a vector instruction has written just before.
__device__ __forceinline__ void load_to_lds(i32x4 rsrc, char* lds, unsigned voff)
{
    const unsigned to = (unsigned)__builtin_amdgcn_readfirstlane((int)(uintptr_t)(__attribute__((address_space(3))) char*)lds);
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(voff), "s"(rsrc) : "memory");
}
__device__ __forceinline__ i32x4 buffer(const char* base, int64_t bytes)
{
    const uint64_t at = (uint64_t)base;
    const unsigned size = (unsigned)(bytes < (int64_t)OUTSIDE ? bytes : (int64_t)OUTSIDE);
    return i32x4{__builtin_amdgcn_readfirstlane((int)(unsigned)at), __builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32 & 0xffff)),
                 __builtin_amdgcn_readfirstlane((int)size), 0x00020000};
}

// ------------------------------------------------------------------------------------------------- the way out
template <int ACT, int COUNT> __device__ __forceinline__ void activate_all(float (&v)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = activate<ACT>(v[i]);
}
template <int COUNT> __device__ __forceinline__ void activate_all(int act, float (&v)[COUNT])
{
    switch (act) {
    case ST_ACT_RELU: activate_all<ST_ACT_RELU>(v); break;
    case ST_ACT_GELU: activate_all<ST_ACT_GELU>(v); break;
    case ST_ACT_GELU_TANH: activate_all<ST_ACT_GELU_TANH>(v); break;
    case ST_ACT_SILU: activate_all<ST_ACT_SILU>(v); break;
    default: break;
    }
}
// COUNT (a multiple of four, or one) values of a row from column n on, of which those below `end` exist: at once, or at the row's end one by one
template <int COUNT> __device__ __forceinline__ void store_run(void* base, int is_bf16, int64_t at, int64_t n, int64_t end, const float (&v)[COUNT])
{
    if (is_bf16) {
        bf16* o = (bf16*)base + at;
        if (n + COUNT <= end) {
            typedef bf16 T __attribute__((ext_vector_type(COUNT)));
            typedef T T2 __attribute__((aligned(2)));
            T u;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) u[i] = (bf16)v[i];
            *(T2*)o = u;
            return;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) if (n + i < end) o[i] = (bf16)v[i];
    } else {
        float* o = (float*)base + at;
        if (n + COUNT <= end) {
            if constexpr (COUNT == 1) *o = v[0];
            else
#pragma unroll
                for (int i = 0; i < COUNT; i += 4) *(f32x4_4*)(o + i) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
            return;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) if (n + i < end) o[i] = v[i];
    }
}
template <int COUNT> __device__ __forceinline__ void load_run(const void* base, int is_bf16, int64_t at, int64_t n, int64_t end, float (&v)[COUNT])
{
    const int there = n + COUNT <= end ? COUNT : (int)(end - n);
    if constexpr (COUNT == 1) v[0] = is_bf16 ? (float)((const bf16*)base)[at] : ((const float*)base)[at];
    else
#pragma unroll
        for (int i = 0; i < COUNT; i += 4) {
            float u[4];
            if (is_bf16) load4((const bf16*)base + at + i, there - i, u); else load4((const float*)base + at + i, there - i, u);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = u[j];
        }
}
// What the sums of row m, columns n .. n + COUNT - 1 (n < p.n) become.  bias: of these columns.
template <int COUNT> __device__ __forceinline__ void finish(const LinearProduct& p, int64_t m, int64_t n, float (&v)[COUNT], const float (&bias)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] += bias[i];
    if (p.pre) store_run(p.pre, p.pre_bf16, m * p.pre_pitch + n, n, p.n, v);
    activate_all(p.act, v);
    if (p.residual) {
        float r[COUNT];
        load_run(p.residual, p.residual_bf16, m * p.residual_pitch + n, n, p.n, r);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] += r[i];
    }
    store_run(p.out, p.out_bf16, m * p.out_pitch + n, n, p.n, v);
}
template <int COUNT> __device__ __forceinline__ void bias_of(const LinearProduct& p, int64_t n, float (&b)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) b[i] = p.bias && n + i < p.n ? p.bias[n + i] : 0.f;
}

// s_waitcnt vmcnt(N) alone; a barrier that memory accesses stay on their side of, without a wait of its own
#define ST_WAIT_VM(N) __builtin_amdgcn_s_waitcnt(((N) & 15) | (((N) >> 4) << 14) | 0x0F70)
#define ST_BARRIER()                    \
    do {                                \
        asm volatile("" ::: "memory");  \
        __builtin_amdgcn_s_barrier();   \
        asm volatile("" ::: "memory");  \
    } while (0)

// ------------------------------------------------------------------------------------------------- an operand's tile
// R rows, loaded by WAVES wavefronts, N blocks of 32 rows of which a wavefront multiplies.
template <class E, bool ALONG, int R, int WAVES, int N> struct Tile;

template <class E, int R, int WAVES, int N> struct Tile<E, true, R, WAVES, N> {
    static constexpr int LOADS = R / 8 / WAVES, READS = N;
    static_assert(WAVES % 2 == 0, "a wavefront's eight rows begin at an even or at an odd multiple of eight in every load");
    i32x4 r;
    unsigned v, step, by, left;     // left: bytes of the row from the lane's chunk on; by: what a turn moves on
    unsigned row;                // of a fragment: its place in the tile
    // stages s0, s0 + every, .. are loaded in turn
    __device__ __forceinline__ Tile(const Operand& o, int64_t row0, int64_t rows, int64_t k, int lane, int wave, int first, int s0, int every)
    {
        const int64_t pitch = o.pitch * sizeof(E);
        const unsigned end = ((unsigned)k * sizeof(E) + 15) / 16 * 16;      // (copies have zeros there)
        r = buffer((const char*)o.p + row0 * pitch, (rows - row0 - 1) * pitch + end);
        const unsigned chunk = ((lane & 7) ^ ((lane >> 4) + 4 * (wave & 1))) * 16 + (unsigned)s0 * STAGE;
        v = (unsigned)(wave * 8 + (lane >> 3)) * (unsigned)pitch + chunk;
        left = end - chunk;
        by = every * STAGE;
        step = WAVES * 8 * (unsigned)pitch;
        row = (unsigned)(first + (lane & 31)) * STAGE;
    }
    __device__ __forceinline__ void load(char* to, int wave)
    {
        unsigned off = v;
        const bool there = (int)left > 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i, off += step) load_to_lds(r, to + (i * WAVES + wave) * 1024, there ? off : OUTSIDE);
        v += by; left -= by;
    }
    __device__ __forceinline__ void fetch(const char* L, int ks, int lane, i32x4 (&f)[N]) const
    {
        const char* at = L + row + ((ks * 2 + (lane >> 5)) ^ (lane >> 1 & 7)) * 16;
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = *(const i32x4*)(at + i * 32 * STAGE);
    }
};

template <class E, int R, int WAVES, int N> struct Tile<E, false, R, WAVES, N> {
    static constexpr int ES = sizeof(E), KS = STAGE / ES, LANES = R * ES / 16, KPI = 64 / LANES;      // a wavefront's load: KPI positions
    static constexpr int LOADS = R / 8 / WAVES, READS = ES == 2 ? 2 * N : 4 * N;
    static_assert(WAVES * KPI % 8 == 0, "the places of a position are the same in every load of a wavefront");
    const char* base; int64_t left, by;      // of the next stage: its first position, and the bytes from there to the matrix's end
    unsigned v, step, at[N];
    static __device__ __forceinline__ unsigned moved(unsigned position)      // by how many chunks
    {
        if constexpr (R == 32) return 0;
        else if constexpr (ES == 4) return 8 * (position >> 2 & 1);
        else if constexpr (R == 64) return 4 * (position >> 1 & 1);
        else return 4 * (position & 3);
    }
    __device__ __forceinline__ Tile(const Operand& o, int64_t row0, int64_t rows, int64_t len, int lane, int wave, int first, int s0, int every)
    {
        const int64_t pitch = o.pitch * ES, from0 = (int64_t)s0 * KS * pitch;
        by = (int64_t)every * KS * pitch;
        base = (const char*)o.p + row0 * ES + from0;
        // (whole chunks: what lies behind the last row inside one is memory that is there)
        left = (len - 1) * pitch + ((rows - row0) * ES + 15) / 16 * 16 - from0;
        const unsigned position = wave * KPI + lane / LANES;
        v = position * (unsigned)pitch + ((lane % LANES) ^ moved(position)) * 16;
        step = WAVES * KPI * (unsigned)pitch;
        const int half = lane >> 5;
        if constexpr (ES == 2) {
            const unsigned from = 8 * half + (lane >> 2 & 3);
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[i] = from * R * 2 + ((first / 8 + i * 4 + 2 * (lane >> 4 & 1) + (lane >> 1 & 1)) ^ moved(from)) * 16 + (lane & 1) * 8;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[i] = 4 * half * R * 4 + (((first + i * 32 + (lane & 31)) / 4) ^ moved(4 * half)) * 16 + (lane & 3) * 4;
        }
    }
    __device__ __forceinline__ void load(char* to, int wave)
    {
        const auto r = buffer(base, left);
        unsigned off = v;
#pragma unroll
        for (int i = 0; i < LOADS; ++i, off += step) load_to_lds(r, to + (i * WAVES + wave) * 1024, off);
        base += by; left -= by;
    }
    __device__ __forceinline__ void fetch(const char* L, int ks, int lane, i32x4 (&f)[N]) const
    {
        (void)lane;
        if constexpr (ES == 2) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                typedef __attribute__((address_space(3))) s16x4* P;
                struct Two { s16x4 lo, hi; } t;
                t.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(L + at[i] + ks * 16 * R * 2));
                t.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(L + at[i] + (ks * 16 + 4) * R * 2));
                f[i] = __builtin_bit_cast(i32x4, t);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) f[i][j] = *(const int*)(L + at[i] + (ks * 8 + j) * R * 4);
        }
    }
};

template <class E> __device__ __forceinline__ Operand second_term(const LinearProduct& p)
{
    return Operand{(const E*)p.a.p + p.a_second, p.a.pitch, p.a.along, p.a.inner};
}

template <class E> __device__ __forceinline__ f32x16 mfma(i32x4 a, i32x4 b, f32x16 c)
{
    if constexpr (sizeof(E) == 2) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else {
        const f32x4 u = __builtin_bit_cast(f32x4, a), v = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(u[j], v[j], c, 0, 0, 0);
        return c;
    }
}

// ------------------------------------------------------------------------------------------------- a block's place
// An XCD gets a run of consecutive tiles, ordered in bands of four tiles of tokens: what its 32 compute units work on at a time is
// 4 x 8 tiles, and less goes from memory to its L2 than with rows of tiles.
struct Place { int second, split, tm, tn; };
__device__ __forceinline__ Place place_of(const GemmPair& pair)
{
    const int second = blockIdx.x >= pair.g[0].blocks;
    const GemmArgs& g = pair.g[second];
    const int block = xcd_band((int)blockIdx.x - (second ? (int)pair.g[0].blocks : 0), (int)g.blocks);
    const int split = __builtin_amdgcn_readfirstlane(fast_quot(block, g.by_tiles));
    const int tile = block - split * (int)g.by_tiles.d;
    const int band = __builtin_amdgcn_readfirstlane(fast_quot(tile, g.by_band)), in_band = tile - band * (int)g.by_band.d;
    const int high = min(BAND, g.tiles_m - band * BAND);
    const int tn = __builtin_amdgcn_readfirstlane(in_band / high);
    return {second, split, band * BAND + in_band - tn * high, tn};
}

// ------------------------------------------------------------------------------------------------- a block's tile
// BM tokens x BN channels a block, WM x WN a wavefront.  Us of a launch with plain epilogue, and what that is:
//   256        8192 tokens 4096 -> 14336   814   1.18 PFLOP/s (the library's plain product 1.40), of which 68 us do not grow with the sums: a
//              block's first loads and its way out, 7 blocks one after the other on a compute unit.  The stages' loads alone take 682 (360 where
//              all of them hit L2), the products alone 670; on operands of zeros, which leave the clock higher, the products take 501 and all of
//              it 654: loads into LDS, and the clock under load.  LDS reads alone take 245
//              both gradients, 8192 tokens 4096 -> 4096   433   1.27 PFLOP/s (the library's 1.17: it turns operands on the way)
//   128        4096 tokens 2048 -> 2048   40   0.86 PFLOP/s, two blocks a compute unit: L2 gives 9 TB/s for its tiles
//   64         2048 tokens 1024 -> 1024   11.3   0.38 PFLOP/s, 16 stages of 0.26 us two a compute unit
//   float32    8192 tokens 4096 -> 4096   1940   0.142 PFLOP/s of the instruction's 0.157 (the library 0.149)
// Tried: 128 x 128 a wavefront, four of them (912 us in the first row's place); stages of 64 bytes, 4 or 5 under way (870); a higher
// wavefront priority around the products (833); a stage's loads spread over the last step's products (834 against 836 with activation, the tiles of 64 and
// 128 1.03 of the time); 256 x 128 tiles (40 shapes of 500 .. 14000 tokens: 1.007 of the time); blocks that stay and ask for their
// next tile's stages before the way out (the same shapes: 1.09, for the registers that takes).
template <class E, int BM, int BN, int WM, int WN, int DEPTH, bool A_ALONG, bool B_ALONG>
__device__ __forceinline__ void product_tile(const GemmArgs& g, char* lds, int64_t m0, int64_t n0, int split, f32x16 (&acc)[WM / 32][WN / 32])
{
    constexpr int WAVES = (BM / WM) * (BN / WN), NA = WN / 32, NB = WM / 32, STEPS = STAGE / 32;
    constexpr int BUF = (BM + BN) * STAGE, MINE = BN * STAGE;       // channels first, then tokens
    const LinearProduct& p = g.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = (int)((int64_t)g.stages * split / g.splits), last = (int)((int64_t)g.stages * (split + 1) / g.splits);
    const int wn = (wave % (BN / WN)) * WN, wm = (wave / (BN / WN)) * WM;
    using Channels = Tile<E, B_ALONG, BN, WAVES, NA>;
    using Tokens = Tile<E, A_ALONG, BM, WAVES, NB>;
    int coming = first < g.once ? first : first - g.once;      // the stage of its term that is loaded next
    Channels channels(p.b, n0, p.n, p.k, lane, wave, wn, coming, 1);
    Tokens tokens(first < g.once ? p.a : second_term<E>(p), m0, p.m, p.k, lane, wave, wm, coming, 1);
    auto next_stage = [&](int buf) {
        if (coming == g.once) {
            coming = 0;
            channels = Channels(p.b, n0, p.n, p.k, lane, wave, wn, 0, 1);
            tokens = Tokens(second_term<E>(p), m0, p.m, p.k, lane, wave, wm, 0, 1);
        }
        ++coming;
        channels.load(lds + buf * BUF, wave);
        tokens.load(lds + buf * BUF + MINE, wave);
    };
    i32x4 a[2][NA], b[2][NB];
    auto fetch = [&](int buf, int ks, int to) {
        channels.fetch(lds + buf * BUF, ks, lane, a[to]);
        tokens.fetch(lds + buf * BUF + MINE, ks, lane, b[to]);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < NA; ++i) acc[j][i] = mfma<E>(a[from][i], b[from][j], acc[j][i]);
    };
    // in the instruction stream: LDS reads spread over the matrix instructions
    auto interleave = [] {
        constexpr int READS = Channels::READS + Tokens::READS, PRODUCTS = NA * NB * (sizeof(E) == 2 ? 1 : 4);
        constexpr int PER = READS > PRODUCTS ? (READS + PRODUCTS - 1) / PRODUCTS : 1;
#pragma unroll
        for (int i = 0; i < (READS + PER - 1) / PER; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
    };
    // DEPTH stages are under way.  A stage's last step has its operands in registers when the barrier is passed; what follows the barrier
    // is the loads of the stage DEPTH later into the buffer that is done with, and the next stage's first operands.  (8192 tokens 4096 -> 14336
    // with the last step's products before the barrier 814 us, behind these loads 828; half stages, twice as many, 870.)
    constexpr int LOADS = Channels::LOADS + Tokens::LOADS;      // of a wavefront and stage
    static_assert((DEPTH - 1) * LOADS < 64, "the counter of loads under way");
    if (first < last) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) if (first + d < last) next_stage(d);
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
        multiply((STEPS - 1) & 1);
        ST_BARRIER();
        if (s + DEPTH < last) next_stage(buf);
        buf = buf + 1 == DEPTH ? 0 : buf + 1;
        if (s + 1 < last) fetch(buf, 0, 0);
    }

}

// Out through LDS, 32 tokens of a wavefront at a time: sums go in four neighbouring channels at a time and come out as runs along a row.
template <int BM, int BN, int WM, int WN, int DEPTH>
__device__ __forceinline__ void tile_out(const GemmArgs& g, char* lds, int64_t m0, int64_t n0, int split, const f32x16 (&acc)[WM / 32][WN / 32])
{
    constexpr int WAVES = (BM / WM) * (BN / WN), PITCH = WN + 4, RUNS = WN / 8, ROWS = 64 / RUNS;
    static_assert(WAVES * 32 * PITCH * 4 <= DEPTH * (BM + BN) * STAGE, "room for the sums");
    const LinearProduct& p = g.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = (wave % (BN / WN)) * WN, wm = (wave / (BN / WN)) * WM;
    const int run = lane % RUNS, row = lane / RUNS, r32 = lane & 31, half = lane >> 5;
    const int64_t n = n0 + wn + run * 8;
    float bias[8];
    bias_of(p, n, bias);
    __syncthreads();
    float* mine = (float*)lds + wave * 32 * PITCH;
#pragma unroll
    for (int j = 0; j < WM / 32; ++j) {
#pragma unroll
        for (int i = 0; i < WN / 32; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4*)(mine + r32 * PITCH + i * 32 + q * 8 + half * 4) =
                    f32x4{acc[j][i][q * 4], acc[j][i][q * 4 + 1], acc[j][i][q * 4 + 2], acc[j][i][q * 4 + 3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int h = 0; h < 32 / ROWS; ++h) {
            const int r = h * ROWS + row;
            const int64_t m = m0 + wm + j * 32 + r;
            const f32x4 lo = *(const f32x4*)(mine + r * PITCH + run * 8), hi = *(const f32x4*)(mine + r * PITCH + run * 8 + 4);
            if (m >= p.m || n >= p.n) continue;
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (g.splits > 1) store_run(p.slabs, 0, ((int64_t)split * p.m + m) * p.n + n, n, p.n, v);
            else finish(p, m, n, v, bias);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// The parts of 32 columns: a column's parts are dealt out to THREADS / 32 threads, whose sums are added in their order.
constexpr int SUM_COLUMNS = 32;
template <int THREADS> __device__ __forceinline__ void sum_columns(const ColumnSums& s, unsigned block, float* lds)
{
    constexpr int GROUPS = THREADS / SUM_COLUMNS;
    const int col = threadIdx.x % SUM_COLUMNS, group = threadIdx.x / SUM_COLUMNS;
    const int64_t i = (int64_t)block * SUM_COLUMNS + col;
    float v = 0.f;
    if (i < s.n)
#pragma unroll 8
        for (int part = group; part < s.n_parts; part += GROUPS) v += s.parts[(int64_t)part * s.n + i];
    lds[threadIdx.x] = v;
    __syncthreads();
    if (group || i >= s.n) return;
    v = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) v += lds[g * SUM_COLUMNS + col];
    s.out[i] = s.accumulate ? s.out[i] + v : v;
}

template <class E, int BM, int BN, int WM, int WN, int DEPTH>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_linear_product(const GemmPair pair)
{
    extern __shared__ __align__(16) char lds[];
    const unsigned both = pair.g[0].blocks + pair.g[1].blocks;
    if (blockIdx.x >= both) { sum_columns<(BM / WM) * (BN / WN) * 64>(pair.sums, blockIdx.x - both, (float*)lds); return; }
    const Place at = place_of(pair);
    const GemmArgs& g = pair.g[at.second];
    const int64_t m0 = (int64_t)at.tm * BM, n0 = (int64_t)at.tn * BN;
    const int split = at.split;
    f32x16 acc[WM / 32][WN / 32] = {};
    if (g.p.a.along) {
        if (g.p.b.along) product_tile<E, BM, BN, WM, WN, DEPTH, true, true>(g, lds, m0, n0, split, acc);
        else product_tile<E, BM, BN, WM, WN, DEPTH, true, false>(g, lds, m0, n0, split, acc);
    } else {
        if (g.p.b.along) product_tile<E, BM, BN, WM, WN, DEPTH, false, true>(g, lds, m0, n0, split, acc);
        else product_tile<E, BM, BN, WM, WN, DEPTH, false, false>(g, lds, m0, n0, split, acc);
    }
    tile_out<BM, BN, WM, WN, DEPTH>(g, lds, m0, n0, split, acc);
}

// ------------------------------------------------------------------------------------------------- small tiles
// 32 tokens x 32 channels a block, for products whose larger tiles would leave compute units without work: latency bounds them, so the
// block's eight wavefronts share the contraction.  Two groups of four take its stages in turn, and of a stage each wavefront one step (two
// LDS reads, one product); the eight sums are added in LDS in their order.
//
// LOOSE: operands at any address with any stride, through registers (a load's 16 bytes may begin anywhere): a chunk that would reach behind a
// row's end is loaded from the row's last 16 bytes and moved to its place, rows and positions that do not exist are zeros.
// (Four stages of a group are under way; eight, in a compute unit's whole LDS, take as long: 64 tokens 512 -> 512 7.4 us and 7.5, 8 tokens
// 4096 -> 4096, weights across, 12.3 and 12.3.)
constexpr int SMALL = SMALL_TILE, SMALL_GROUPS = 2, SMALL_BUF = 2 * SMALL * STAGE, SMALL_THREADS = SMALL_GROUPS * 256;
constexpr size_t small_lds(bool loose)
{
    const size_t stages = (size_t)SMALL_GROUPS * (loose ? 2 : 4) * SMALL_BUF, sums = (size_t)SMALL_THREADS / 64 * SMALL * (SMALL + 4) * 4;
    return stages > sums ? stages : sums;
}

template <class E, bool ALONG> struct LooseTile {
    static constexpr int CH = 16 / sizeof(E), KS = STAGE / sizeof(E);
    using Chunk = Run<E, CH>;
    const E* base; int64_t pitch, k;      // k: positions of the contraction that can be read
    int once; int64_t second;             // stages of a term; from a term to the next
    int position;                // of the chunk in a stage's contraction
    int down;                    // across: by how much the row's last chunk is moved; along: nothing
    __device__ __forceinline__ LooseTile(const Operand& o, int64_t row0, int64_t rows, int64_t len, int lane, int wave, int once_, int64_t second_)
        : once(once_), second(second_)
    {
        pitch = o.pitch; k = ALONG ? o.inner : len;
        if constexpr (ALONG) {
            position = ((lane & 7) ^ ((lane >> 4) + 4 * (wave & 1))) * CH;
            base = (const E*)o.p + std::min<int64_t>(row0 + wave * 8 + (lane >> 3), rows - 1) * pitch;
            down = 0;
        } else {
            constexpr int LANES = SMALL / CH;
            position = wave * (64 / LANES) + lane / LANES;
            const int64_t at = row0 + (lane % LANES) * CH, from = std::min(at, o.inner - CH);
            base = (const E*)o.p + from;
            down = (int)std::min<int64_t>(at - from, CH);
        }
    }
    __device__ __forceinline__ void load(int s, Chunk& c) const
    {
        const int64_t at = (int64_t)(s < once ? s : s - once) * KS + position;
        c.load((ALONG ? base + std::min(at, k - CH) : base + std::min(at, k - 1) * pitch) + (s < once ? 0 : second));
    }
    __device__ __forceinline__ void store(int s, Chunk& c, char* to) const      // to: the lane's place
    {
        if (s >= once) s -= once;
        const int64_t at = (int64_t)s * KS + position;
        if constexpr (ALONG) {
            if (((int64_t)s + 1) * KS > k) { const int64_t d = at - (k - CH); if (d > 0) c.down((int)std::min<int64_t>(d, CH)); }
        } else {
            if (down) c.down(down);
            if (at >= k) c.down(CH);
        }
        *(i32x4*)to = __builtin_bit_cast(i32x4, c);
    }
};

template <class E, bool A_ALONG, bool B_ALONG, bool LOOSE>
__device__ __forceinline__ void small_tile(const GemmArgs& g, char* lds, int64_t m0, int64_t n0, int split, f32x16& acc)
{
    constexpr int DEPTH = LOOSE ? 2 : 4, AHEAD = 4;
    const LinearProduct& p = g.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave >> 2, w4 = wave & 3;
    const int first = (int)((int64_t)g.stages * split / g.splits), last = (int)((int64_t)g.stages * (split + 1) / g.splits);
    const int turns = (last - first + SMALL_GROUPS - 1) / SMALL_GROUPS;
    char* const own = lds + group * DEPTH * SMALL_BUF;
    auto stage_of = [&](int turn) { return first + turn * SMALL_GROUPS + group; };
    using Channels = Tile<E, B_ALONG, SMALL, 4, 1>;
    using Tokens = Tile<E, A_ALONG, SMALL, 4, 1>;
    bool in_second = first + group >= g.once;
    const int begin = first + group - (in_second ? g.once : 0);
    Channels channels(p.b, n0, p.n, p.k, lane, w4, 0, begin, SMALL_GROUPS);
    Tokens tokens(in_second ? second_term<E>(p) : p.a, m0, p.m, p.k, lane, w4, 0, begin, SMALL_GROUPS);
    auto multiply = [&](const char* buf) {
        i32x4 a[1], b[1];
        channels.fetch(buf, w4, lane, a);
        tokens.fetch(buf + SMALL * STAGE, w4, lane, b);
        acc = mfma<E>(a[0], b[0], acc);
    };
    if constexpr (LOOSE) {
        const LooseTile<E, B_ALONG> from_b(p.b, n0, p.n, p.k, lane, w4, g.once, 0);
        const LooseTile<E, A_ALONG> from_a(p.a, m0, p.m, p.k, lane, w4, g.once, p.a_second);
        typename LooseTile<E, true>::Chunk c[AHEAD][2];
        auto ask = [&](int turn, int u) { if (stage_of(turn) < last) { from_b.load(stage_of(turn), c[u][0]); from_a.load(stage_of(turn), c[u][1]); } };
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) ask(u, u);
        for (int t = 0; t < turns; t += AHEAD)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (t + u >= turns) break;
                char* const buf = own + (u & 1) * SMALL_BUF;
                const int s = stage_of(t + u);
                if (s < last) {
                    from_b.store(s, c[u][0], buf + threadIdx.x % 256 * 16);
                    from_a.store(s, c[u][1], buf + SMALL * STAGE + threadIdx.x % 256 * 16);
                }
                ask(t + u + AHEAD, u);
                __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0)
                ST_BARRIER();
                if (s < last) multiply(buf);
            }
    } else {
        auto ask = [&](int turn) {
            const int s = stage_of(turn);
            if (s >= last) return;
            if (!in_second && s >= g.once) {
                in_second = true;
                channels = Channels(p.b, n0, p.n, p.k, lane, w4, 0, s - g.once, SMALL_GROUPS);
                tokens = Tokens(second_term<E>(p), m0, p.m, p.k, lane, w4, 0, s - g.once, SMALL_GROUPS);
            }
            char* const buf = own + turn % DEPTH * SMALL_BUF;
            channels.load(buf, w4);
            tokens.load(buf + SMALL * STAGE, w4);
        };
#pragma unroll
        for (int t = 0; t < DEPTH - 1; ++t) ask(t);
        for (int t = 0; t < turns; ++t) {
            // this stage is there (two loads of each of the DEPTH - 2 behind it may be on their way), and the one before is read
            if (stage_of(t + DEPTH - 2) < last) ST_WAIT_VM(2 * (DEPTH - 2)); else ST_WAIT_VM(0);
            __builtin_amdgcn_s_waitcnt(0xc07f);
            ST_BARRIER();
            ask(t + DEPTH - 1);
            if (stage_of(t) < last) multiply(own + t % DEPTH * SMALL_BUF);
        }
    }
}

__device__ __forceinline__ void small_out(const GemmArgs& g, char* lds, int64_t m0, int64_t n0, int split, const f32x16& acc)
{
    const LinearProduct& p = g.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __syncthreads();
    constexpr int PITCH = SMALL + 4;
    float* const sums = (float*)lds;
    const int r32 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *(f32x4*)(sums + (wave * SMALL + r32) * PITCH + q * 8 + half * 4) = f32x4{acc[q * 4], acc[q * 4 + 1], acc[q * 4 + 2], acc[q * 4 + 3]};
    __syncthreads();
    const int run = threadIdx.x & 7, row = threadIdx.x >> 3;
    const int64_t m = m0 + row, n = n0 + run * 4;
    if (row >= SMALL || m >= p.m || n >= p.n) return;
    float v[4] = {}, bias[4];
    bias_of(p, n, bias);
#pragma unroll
    for (int w = 0; w < SMALL_GROUPS * 4; ++w) {
        const f32x4 u = *(const f32x4*)(sums + (w * SMALL + row) * PITCH + run * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u[e];
    }
    if (g.splits > 1) store_run(p.slabs, 0, ((int64_t)split * p.m + m) * p.n + n, n, p.n, v);
    else finish(p, m, n, v, bias);
}

template <class E, bool LOOSE> __global__ __launch_bounds__(SMALL_THREADS) void k_linear_small(const GemmPair pair)
{
    extern __shared__ __align__(16) char lds[];
    const unsigned both = pair.g[0].blocks + pair.g[1].blocks;
    if (blockIdx.x >= both) { sum_columns<SMALL_THREADS>(pair.sums, blockIdx.x - both, (float*)lds); return; }
    const Place at = place_of(pair);
    const GemmArgs& g = pair.g[at.second];
    const int64_t m0 = (int64_t)at.tm * SMALL, n0 = (int64_t)at.tn * SMALL;
    f32x16 acc = {};
    if (g.p.a.along) {
        if (g.p.b.along) small_tile<E, true, true, LOOSE>(g, lds, m0, n0, at.split, acc);
        else small_tile<E, true, false, LOOSE>(g, lds, m0, n0, at.split, acc);
    } else {
        if (g.p.b.along) small_tile<E, false, true, LOOSE>(g, lds, m0, n0, at.split, acc);
        else small_tile<E, false, false, LOOSE>(g, lds, m0, n0, at.split, acc);
    }
    small_out(g, lds, m0, n0, at.split, acc);
}

// The slabs of split products, added in one order, and what the product's own way out does otherwise: runs of COUNT of a row.  GROUPS threads
// share a run where there are few of them, each with some of the slabs.
template <int GROUPS, int COUNT> __global__ __launch_bounds__(256) void k_linear_join(const GemmPair pair, int64_t first, int64_t all)
{
    __shared__ float sums[GROUPS > 1 ? GROUPS * (256 / GROUPS) * COUNT : 1];
    constexpr int EACH = 256 / GROUPS;
    const int group = threadIdx.x / EACH, mine = threadIdx.x % EACH;
    for (int64_t base = (int64_t)blockIdx.x * EACH; base < all; base += (int64_t)gridDim.x * EACH) {
        const int64_t i = base + mine < all ? base + mine : all - 1;
        const bool second = i >= first;
        const GemmArgs& g = pair.g[second];
        const LinearProduct& p = g.p;
        const int64_t runs = (p.n + COUNT - 1) / COUNT, at = second ? i - first : i, m = at / runs, n = (at - m * runs) * COUNT, size = p.m * p.n;
        float v[COUNT] = {};
        const float* from = p.slabs + m * p.n + n;
#pragma unroll 4
        for (int s = group; s < g.splits; s += GROUPS) {
            float u[COUNT];
            load_run(from + s * size, 0, 0, n, p.n, u);
#pragma unroll
            for (int e = 0; e < COUNT; ++e) v[e] += u[e];
        }
        if constexpr (GROUPS > 1) {
            __syncthreads();      // (the turn before has been read)
#pragma unroll
            for (int e = 0; e < COUNT; ++e) sums[(group * COUNT + e) * EACH + mine] = v[e];
            __syncthreads();
            if (group) continue;
#pragma unroll
            for (int e = 0; e < COUNT; ++e) {
                v[e] = 0.f;
#pragma unroll
                for (int q = 0; q < GROUPS; ++q) v[e] += sums[(q * COUNT + e) * EACH + mine];
            }
        }
        if (base + mine >= all) continue;
        float bias[COUNT];
        bias_of(p, n, bias);
        finish(p, m, n, v, bias);
    }
}

// --------------------------------------------------------------------------------------------------- few tokens
// Up to 32 tokens, the weights along the contraction: they are read once, 16 bytes a lane straight from memory into matrix instructions of
// 16 channels x 16 tokens (v_mfma_f32_16x16x32_bf16: lane l supplies A[l % 16][8*(l/16) .. +7] and B[8*(l/16) .. +7][l % 16] and receives
// D[4*(l/16) + r][l % 16]; v_mfma_f32_16x16x4_f32: one value of a lane's 16 bytes an instruction).  A block takes 16 channels, each of its
// eight wavefronts an eighth of the contraction; the eighths are added in LDS in their order.  Rows may begin at any address; the last
// chunks of a row, those that would reach behind it, are loaded value by value.  Bytes bound it: 1 token 2048 -> 5632 6 us (23 MB, 3.9 TB/s), 12 tokens
// 4096 -> 4096 8 us (34 MB, 4.2 TB/s); twice as many loads under way, with twice the registers, take 0.6 us longer.
constexpr int FEW_WAVES = 8;
struct FewArgs { LinearProduct p; int64_t x_row, x_step; int per_wave; };       // per_wave: bytes, a multiple of 64

template <class E> __device__ __forceinline__ i32x4 load_any(const char* p)
{
    if constexpr (sizeof(E) == 2) return __builtin_bit_cast(i32x4, *(const u32x4_2*)p);
    else return __builtin_bit_cast(i32x4, *(const f32x4_4*)p);
}
// `there` values (0 .. 16 / sizeof(E)), `step` values apart, zeros behind them
template <class E> __device__ __forceinline__ i32x4 load_some(const char* p, int there, int64_t step)
{
    i32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 2) {
            const unsigned short* u = (const unsigned short*)p;
            const unsigned lo = 2 * i < there ? u[2 * i * step] : 0u, hi = 2 * i + 1 < there ? u[(2 * i + 1) * step] : 0u;
            v[i] = (int)(lo | hi << 16);
        } else v[i] = i < there ? ((const int*)p)[i * step] : 0;
    }
    return v;
}
template <class E> __device__ __forceinline__ f32x4 mfma16(i32x4 a, i32x4 b, f32x4 c)
{
    if constexpr (sizeof(E) == 2) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else {
        const f32x4 u = __builtin_bit_cast(f32x4, a), v = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(u[j], v[j], c, 0, 0, 0);
        return c;
    }
}

template <class E, int NT> __global__ __launch_bounds__(FEW_WAVES * 64) void k_linear_few(const FewArgs f)
{
    constexpr int ES = sizeof(E), AHEAD = 4;
    __shared__ __align__(16) float part[FEW_WAVES * NT * 256];
    const LinearProduct& p = f.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t end = p.k * ES, whole = end / 64 * 64;
    const int64_t from = (int64_t)wave * f.per_wave, to = std::min(from + f.per_wave, end), to_whole = std::min(to, whole);
    const int64_t off = (lane >> 4) * 16;
    const char* w = (const char*)p.b.p + std::min(n0 + (lane & 15), p.n - 1) * p.b.pitch * ES + off;      // (what is beyond the channels or the tokens is not used)
    const char* x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = (const char*)p.a.p + std::min<int64_t>(t * 16 + (lane & 15), p.m - 1) * f.x_row * ES + off * f.x_step;
    f32x4 acc[NT] = {};
    int64_t k = from;
    if (f.x_step == 1) {
        for (; k + AHEAD * 64 <= to_whole; k += AHEAD * 64) {
            i32x4 a[AHEAD], b[AHEAD][NT];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                a[u] = load_any<E>(w + k + u * 64);
#pragma unroll
                for (int t = 0; t < NT; ++t) b[u][t] = load_any<E>(x[t] + k + u * 64);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t] = mfma16<E>(a[u], b[u][t], acc[t]);
        }
        for (; k < to_whole; k += 64) {
            const i32x4 a = load_any<E>(w + k);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma16<E>(a, load_any<E>(x[t] + k), acc[t]);
        }
    }
    for (; k < to; k += 64) {      // the end of the rows, or tokens that lie across memory
        const int there = (int)std::max<int64_t>(0, std::min<int64_t>(16, end - k - off)) / ES;
        const i32x4 a = there == 16 / ES ? load_any<E>(w + k) : load_some<E>(w + k, there, 1);
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = mfma16<E>(a, load_some<E>(x[t] + k * f.x_step, there, f.x_step), acc[t]);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) *(f32x4*)(part + (wave * NT + t) * 256 + (lane & 15) * 16 + (lane >> 4) * 4) = acc[t];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 256; i += FEW_WAVES * 64) {
        const int64_t m = i >> 4, n = n0 + (i & 15);
        if (m >= p.m || n >= p.n) continue;
        float v[1] = {0.f}, bias[1];
        bias_of(p, n, bias);
#pragma unroll
        for (int u = 0; u < FEW_WAVES; ++u) v[0] += part[u * NT * 256 + i];
        finish(p, m, n, v, bias);
    }
}

// Where a wavefront's eighth of a row is short, or the tokens are so few that reading them in every block does not count.  Against the tiles, us a
// call: 1 token 3000 -> 2000 6.7 and 9.8, 8 tokens 4096 -> 4096 9.3 and 12.5, 20 11.9 and 12.9, 16 tokens 1024 -> 12000 8.1 and 9.0; but 16 tokens
// 4096 -> 14336 37 and 28, 8192 -> 1000 16.7 and 10.6, 32 tokens 4096 -> 4096 13.4 and 12.8.  Rows of bfloat16 at odd addresses, whose 16 bytes the
// card fetches in pieces: 16 tokens 1001 -> 3001 7.3 and 7.7, 20 8.5 and 7.6, 20 tokens 4097 -> 4097 51 and 19.  float32: 16 tokens 2048 -> 5632 17.1
// and 19.4, 8 tokens 4096 -> 4096 14.5 and 23.1, 16 tokens 4096 -> 14336 67 and 56, 32 tokens 8192 -> 500 43 and 12.
// Beyond 4096, weights that no cache holds, 1, 4, 8 and 16 tokens here against one time of the tiles (which hardly depends on the tokens), a call in a graph:
// 5632 -> 2048 10.8, 11.5, 12.3, 14.3 and 11.9; 8192 -> 1024 13.7 - 18.4 and 11.2; 16384 -> 500 24.7 - 33.7 and 11.8; 14336 -> 4096 29.2, 31.2, 32.7, 37.7 and
// 29.1; 8192 -> 8192 29.0, 31.5, 34.8, 41.0 and 33.3: a tenth to be had for one token of some shapes, twice the time to be lost in others.  float32, 1
// token: 5632 -> 2048 19.1 and 19.0, 14336 -> 4096 51 and 62.  At odd addresses, 1, 4 and 8 tokens: 1001 -> 3001 5.5, 6.6, 6.8 and 7.3, 8.9, 8.5; 2049 -> 2049 9.2, 11.6,
// 12.7 and 14.0, 15.1, 15.0; 4097 -> 4097 17.9, 27.1, 31.0 and 24.0, 25.4, 25.3; 14337 -> 1001 47.9, 64.6, 72.1 and 17.2, 18.3, 18.3: the limit of 1024 keeps clear of
// what is lost at long rows and leaves up to a third at 1025 .. 4096 with few tokens.  Tokens that lie column by column, whose values are loaded one by one: 8 tokens
// 1024 -> 4096 6.8 and 6.8, 4096 -> 4096 21.5 and 14.4, which the rule does not tell apart.
bool linear_few(int64_t m, int64_t n, int64_t k, int is_bf16, bool aligned)
{
    if (m > 32 || k > 4096) return false;
    if (is_bf16) return aligned ? m <= 8 || (m <= 20 && (n <= 4096 || k <= 1024)) : m <= 16 && k <= 1024;
    return k <= 2048 || m <= 8 || (m <= 20 && n >= 2000 && n <= 8192);
}
template <class E> static void few_launch(Ctx& c, const FewArgs& f)
{
    const dim3 grid((unsigned)ceil_div(f.p.n, 16));
    if (f.p.m <= 16) ST_LAUNCH(c, "linear_few", (k_linear_few<E, 1>), grid, dim3(FEW_WAVES * 64), 0, f);
    else ST_LAUNCH(c, "linear_few", (k_linear_few<E, 2>), grid, dim3(FEW_WAVES * 64), 0, f);
}
void linear_product_few(Ctx& c, const LinearProduct& p, int is_bf16)
{
    const int64_t es = is_bf16 ? 2 : 4;
    const FewArgs f{p, p.a.along ? p.a.pitch : 1, p.a.along ? 1 : p.a.pitch, (int)round_up(ceil_div(p.k * es, FEW_WAVES), 64)};
    if (is_bf16) few_launch<bf16>(c, f); else few_launch<float>(c, f);
}

// --------------------------------------------------------------------------------------- choice of tile and split
// What a call is estimated to take, us: a stage of 128 bytes of a tile takes `stage` of a compute unit's time (as much where it is alone as
// where two blocks share the unit's throughput), a block `block` to begin and to end; half of what blocks leave idle that do not divide among 256
// compute units is lost; parts of a split contraction cost a join, copies of odd operands a launch and their bytes.  Fitted to 140 forward and
// backward calls of 33 .. 12000 tokens, 96 .. 14336 channels, each with every tile and 1 .. 16 splits: what it chooses takes 1.03 (float32 1.04) times
// the best of them, geometric mean, where thresholds on the number of tiles took 1.06 (1.13).
struct TileCost { int tile; double stage[2], block[2]; };      // float32, bfloat16
constexpr TileCost TILE_COSTS[] = {{SMALL, {0.20, 0.13}, {1.0, 1.0}}, {64, {0.64, 0.26}, {0.6, 0.6}}, {128, {2.24, 0.57}, {1.5, 1.0}}, {256, {8.2, 1.72}, {5.0, 5.0}}};
constexpr double JOIN_US = 4.0, JOIN_BYTE_US = 3e-7, COPY_US = 1.5, COPY_BYTE_US = 4e-7;
constexpr int MOST_SPLITS = 32, LEAST_STAGES = 8;
LinearForm linear_form(const Extent* e, int count, int is_bf16, int64_t copied, bool prepared)
{
    LinearForm best = {64, {1, 1}};
    double least = 1e300;
    int64_t stages[2] = {1, 1}, longest = 1;
    for (int i = 0; i < count; ++i) { stages[i] = ceil_div(e[i].k * (is_bf16 ? 2 : 4), STAGE); longest = std::max(longest, stages[i]); }
    for (const TileCost& c : TILE_COSTS) {
        int64_t tiles[2] = {0, 0};
        for (int i = 0; i < count; ++i) tiles[i] = ceil_div(e[i].m, c.tile) * ceil_div(e[i].n, c.tile);
        const double stage = c.stage[is_bf16], block = c.block[is_bf16];
        for (int64_t s = 1; s <= MOST_SPLITS && (s == 1 || longest >= LEAST_STAGES * s); s *= 2) {
            LinearForm f = {c.tile, {1, 1}};
            double work = 0, alone = 0, slabs = 0;
            int64_t blocks = 0;
            bool joined = false;
            for (int i = 0; i < count; ++i) {
                const int64_t k = std::max<int64_t>(1, std::min(s, stages[i] * s / longest));
                f.splits[i] = (int)k;
                work += (double)(tiles[i] * stages[i]);
                blocks += tiles[i] * k;
                alone = std::max(alone, (double)(ceil_div(stages[i], k) * ceil_div(tiles[i] * k, c.tile == 256 ? 256 : 512)) * stage);
                if (k > 1) { joined = true; slabs += (double)e[i].m * e[i].n * k * 4; }
            }
            if (c.tile == SMALL && blocks > 2048) continue;      // (43 tokens, gradients of 1601 -> 2582: 4233 of them, 28 us, 128 x 128 13)
            const double rounds = (double)ceil_div(blocks, 256), idle = rounds * 256 / blocks - 1;
            const double us = std::max(work * stage / 256 * (1 + 0.5 * idle) + rounds * block, alone + block) + (joined ? JOIN_US + slabs * JOIN_BYTE_US : 0)
                              + (c.tile != SMALL && copied ? (prepared ? 0 : COPY_US) + copied * COPY_BYTE_US : 0);
            if (us < least) { least = us; best = f; }
        }
    }
    return best;
}

template <class E, int BM, int BN, int WM, int WN, int DEPTH>
static void launch(Ctx& c, const GemmPair& g)
{
    constexpr size_t lds = (size_t)DEPTH * (BM + BN) * STAGE;
    constexpr int threads = (BM / WM) * (BN / WN) * 64;
    ensure_dynamic_lds((const void*)k_linear_product<E, BM, BN, WM, WN, DEPTH>, lds);
    constexpr const char* name = BM == 256 ? "linear_product_256" : BM == 64 ? "linear_product_64" : DEPTH > 2 ? "linear_product_128_deep" : "linear_product_128";
    const unsigned grid = g.g[0].blocks + g.g[1].blocks + (unsigned)ceil_div(g.sums.n, SUM_COLUMNS);
    ST_LAUNCH(c, name, (k_linear_product<E, BM, BN, WM, WN, DEPTH>), dim3(grid), dim3(threads), lds, g);
}
template <class E, bool LOOSE> static void launch_small(Ctx& c, const GemmPair& g)
{
    ensure_dynamic_lds((const void*)k_linear_small<E, LOOSE>, small_lds(LOOSE));
    const dim3 grid(g.g[0].blocks + g.g[1].blocks + (unsigned)ceil_div(g.sums.n, SUM_COLUMNS));
    ST_LAUNCH(c, LOOSE ? "linear_small_loose" : "linear_small", (k_linear_small<E, LOOSE>), grid, dim3(SMALL_THREADS), small_lds(LOOSE), g);
}
// 128 x 128 with four stages under way takes a compute unit's LDS, with two a half.  Up to 256 blocks each has a unit for itself; beyond, two side by side are worth
// more than the depth.  Four stages and two, us: bfloat16 135 blocks (3384 tokens 1416 -> 584) 19.8 and 25.5, 184 (408 tokens 3088 -> 5784) 36.0 and 48.7, 230 (5824
// tokens 5976 -> 520) 76 and 98; 264 blocks (992 tokens 216 -> 4176) 15.4 and 11.1, 288 (2296 tokens 3008 -> 2024) 57 and 41, 550 (6976 tokens 2144 -> 1200) 72 and 70.
// float32, whose products take longer than loads: 207 - 252 blocks 0.98 - 1.00 of the deep one's time either way, 410 - 684 blocks 0.88 - 0.95.
template <class E> static void launch_tile(Ctx& c, const GemmPair& g, int tile)
{
    if (tile == SMALL) {
        if (g.g[0].p.loose || g.g[1].p.loose) launch_small<E, true>(c, g); else launch_small<E, false>(c, g);
    } else if (tile == 256) launch<E, 256, 256, 128, 64, 2>(c, g);
    else if (tile == 128 && g.g[0].blocks + g.g[1].blocks <= 256) launch<E, 128, 128, 64, 32, 4>(c, g);
    else if (tile == 128) launch<E, 128, 128, 64, 32, 2>(c, g);
    else launch<E, 64, 64, 32, 32, 4>(c, g);
}

void linear_products(Ctx& c, const LinearProduct* p, int count, const LinearForm& f, int is_bf16, const ColumnSums& sums)
{
    if (count == 0 && sums.n == 0) return;
    GemmPair g{}, joined{};
    g.sums = sums;
    int n_joined = 0;
    int64_t cells[2] = {0, 0};
    for (int i = 0; i < count; ++i) {
        const int64_t tm = ceil_div(p[i].m, f.tile), tn = ceil_div(p[i].n, f.tile);
        const int once = (int)ceil_div(p[i].k * (is_bf16 ? 2 : 4), STAGE);
        g.g[i] = GemmArgs{p[i], fast_div((int)(tm * tn)), fast_div((int)(tn * BAND)), (int)tm, f.splits[i],
                          p[i].a_second ? 2 * once : once, once, (unsigned)(tm * tn * f.splits[i])};
        if (f.splits[i] > 1) { cells[n_joined] = p[i].m; joined.g[n_joined++] = g.g[i]; }
    }
    if (is_bf16) launch_tile<bf16>(c, g, f.tile); else launch_tile<float>(c, g, f.tile);
    if (n_joined) {
        // (few runs: eight threads share one)
        auto runs = [&](int i, int count) { return cells[i] ? cells[i] * ceil_div(joined.g[i].p.n, count) : 0; };
        const bool few = runs(0, 8) + runs(1, 8) < 1 << 16;
        const int count = few ? 4 : 8;
        const int64_t first = runs(0, count), all = first + runs(1, count), blocks = ceil_div(all, few ? 32 : 256);
        const dim3 grid((unsigned)(blocks > 8192 ? 8192 : blocks));
        if (few) ST_LAUNCH(c, "linear_join", (k_linear_join<8, 4>), grid, dim3(256), 0, joined, first, all);
        else ST_LAUNCH(c, "linear_join", (k_linear_join<1, 8>), grid, dim3(256), 0, joined, first, all);
    }
}

}  // namespace st
