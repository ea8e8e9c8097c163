// Rows of float matrices as 8-bit integers with a scale each, and the sums of a gradient's rows.
//
//   a = max |x_k|,  scale = a * (1/127),  q_k = rint(x_k * (127 * (1/a))),  each operation rounded to float32.
//
// Largest values are found on the bit patterns of |x| as unsigned numbers: the order is that of the values, and an infinity or a NaN comes
// out on top, where a floating-point maximum would lose the NaN.  One float32 division per row, then a product and a rounding per value;
// the rounding is an addition of 1.5 * 2^23, whose low byte then is the code in two's complement.
//
// A call's sources go through two launches at most.  The first quantises the sources whose rows lie along memory, each row read once; of
// a source that is to be transposed it finds the largest value (and the sum) of each row's parts.  The second transposes those through
// LDS as codes.  (Sources that share a launch do not wait for one another: a backward pass has four, of which some are a few tiles.)
#include "st_quantize.hpp"

#include <algorithm>
#include <type_traits>

namespace st {

struct Job {
    const void *x, *mask;
    int64_t pitch, mask_pitch, rows, len, q_pitch, per_part;
    int8_t* q;
    float *scale, *sum, *part_max, *part_sum;
    int parts;
    unsigned len_tiles, tiles_each, len_blocks;      // second launch: tiles of 128 positions, of a block, blocks of a row of tiles
    uint8_t bf16_, mask_bf16, along;
};
struct Jobs { unsigned first1[4], first2[4]; int n; Job job[4]; };      // first block of each job in the two launches

template <class M, class T, int COUNT, class F> __device__ __forceinline__ void clear_masked(const M* row, int len, F at, Raw8<T> (&v)[COUNT])
{
    Raw8<M> on[COUNT];
    load_row(row, len, at, on);
#pragma unroll
    for (int k = 0; k < COUNT; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) if (!(on[k][i] > 0.f)) v[k].clear(i);
}
template <class T> __device__ __forceinline__ float sum8(const Raw8<T>& v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

struct Shared {
    union {
        struct { unsigned tops[4]; double sums[4]; } rows;
        struct { unsigned tops[32][64]; float sums[32][64]; } parts;
        struct { unsigned tops[4][64]; double sums[4][64]; float mult[64]; unsigned tile[2][64][33]; } turn;   // 33: rows begin on other banks
    };
};

// ------------------------------------------------------------------------------------ rows that lie along memory
// LANES threads a row.  A thread holds KEEP runs of eight values of its row, as they came, between the search for the largest and the
// rounding, so a row of up to 8 * KEEP * LANES values is read once; longer rows read the rest twice.  A wavefront takes a row of up to 4096
// bfloat16 values by itself: no barrier, eight loads under way.  Bytes bound it: 8192 x 4096 bfloat16 in 19 us, 5.3 TB/s.
template <class T, int LANES, int KEEP, bool NT = false> __device__ __forceinline__ void rows_role(const Job& j, unsigned block, Shared& sh)
{
    constexpr int MORE = 4;      // runs under way beyond those
    const int lane = threadIdx.x % LANES;
    int64_t row = (int64_t)block * (256 / LANES) + threadIdx.x / LANES;
    const bool there = row < j.rows;
    row = there ? row : j.rows - 1;      // (what a thread without a row finds is not used)
    const int len = (int)j.len;
    const T* x = (const T*)j.x + row * j.pitch;
    unsigned top = 0;
    double total = 0.0;
    auto load = [&](auto at, auto& v) {
        load_row<NT>(x, len, at, v);
        if (!j.mask) return;
        if (j.mask_bf16) clear_masked((const bf16*)j.mask + row * j.mask_pitch, len, at, v);
        else clear_masked((const float*)j.mask + row * j.mask_pitch, len, at, v);
    };
    auto see = [&](const Raw8<T>& v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[i]));
        if (j.sum) total += sum8(v);
    };
    Raw8<T> v[KEEP];
    load([&](int k) { return (k * LANES + lane) * 8; }, v);
#pragma unroll
    for (int k = 0; k < KEEP; ++k) see(v[k]);
    for (int at = (KEEP * LANES + lane) * 8; at < len; at += MORE * LANES * 8) {
        Raw8<T> w[MORE];
        load([&](int k) { return at + k * LANES * 8; }, w);
#pragma unroll
        for (int k = 0; k < MORE; ++k) see(w[k]);
    }
    if (j.sum) {
#pragma unroll
        for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) total += __shfl_xor(total, d);
        if (LANES == 256) {
            if ((threadIdx.x & 63) == 0) sh.rows.sums[threadIdx.x >> 6] = total;
            __syncthreads();
            total = (sh.rows.sums[0] + sh.rows.sums[1]) + (sh.rows.sums[2] + sh.rows.sums[3]);
        }
        if (there && lane == 0) j.sum[row] = (float)total;
    }
    if (!j.q) return;
    top = LANES == 32 ? half_max(top) : wave_max(top);
    if (LANES == 256) {
        if ((threadIdx.x & 63) == 0) sh.rows.tops[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(sh.rows.tops[0], sh.rows.tops[1]), max(sh.rows.tops[2], sh.rows.tops[3]));
    }
    if (!there) return;
    float s;
    const float r = row_multiplier(top, &s);
    if (lane == 0) j.scale[row] = s;
    const int64_t padded = (j.len + OPERAND_QUANTUM - 1) / OPERAND_QUANTUM * OPERAND_QUANTUM;
    const int end = (int)(padded < j.q_pitch ? padded : j.q_pitch);
    int8_t* qr = j.q + row * j.q_pitch;
    auto put = [&](int at, const Raw8<T>& w) {
        if (at >= end) return;      // (pitch and quantum are multiples of 8: a run is written whole or not at all)
        *(uint2*)(qr + at) = make_uint2(pack4(code_of(w[0], r), code_of(w[1], r), code_of(w[2], r), code_of(w[3], r)),
                                        pack4(code_of(w[4], r), code_of(w[5], r), code_of(w[6], r), code_of(w[7], r)));
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k) v[k].repack();
#pragma unroll
    for (int k = 0; k < KEEP; ++k) put((k * LANES + lane) * 8, v[k]);
    for (int at = (KEEP * LANES + lane) * 8; at < end; at += MORE * LANES * 8) {
        Raw8<T> w[MORE];
        load([&](int k) { return at + k * LANES * 8; }, w);
#pragma unroll
        for (int k = 0; k < MORE; ++k) put(at + k * LANES * 8, w[k]);
    }
}
template <class T> constexpr int row_keep() { return sizeof(T) == 2 ? 8 : 4; }
static __host__ __device__ __forceinline__ int row_lanes(int64_t len, int is_bf16) { return len <= 1024 ? 32 : len <= (is_bf16 ? 4096 : 2048) ? 64 : 256; }

// --------------------------------------------------------------------------------------- rows that lie across it
// The source is a matrix [len][pitch] whose columns are the operand's rows.  A thread takes 16 bytes of a position, so that 64 columns of
// it are eight (bfloat16) or sixteen (float32) threads and whole lines of memory are read.  Bytes bound both launches where there are many:
// a backward pass of 8192 tokens 4096 -> 4096 in bfloat16 with a mask, 75 us (403 MB, 5.4 TB/s) and 52 (322 MB, 6.2); where there are few,
// 4 to 5 us each, a chain of launch, loads, LDS and stores.
template <class T> constexpr int across() { return 16 / (int)sizeof(T); }              // columns of a thread
template <class T> constexpr int groups() { return 4 * across<T>(); }                  // positions a block takes at once

// A run of a position and what masks it, on their way; settle() before they are used.
struct Columns { int64_t col, from, rows; int down; };      // of a thread: its first, where its runs are loaded from, how far they are moved
template <class T> __device__ __forceinline__ Columns columns_of(int64_t col, int64_t rows)
{
    constexpr int V = across<T>();
    const int64_t from = run_start<V, int64_t>(col, rows), d = col - from;
    return Columns{col, from, rows, d < V ? (int)d : V};
}
template <class T, class M, bool SHORT, bool NT> struct Masked {
    static constexpr int V = across<T>();
    Run<T, V> x;
    Run<M, V> m;
    __device__ __forceinline__ void load(const Job& j, int64_t line, const Columns& c)
    {
        const int n = SHORT && c.col < c.rows ? (int)(c.rows - c.col) : 0;
        if constexpr (SHORT) x.load_short((const T*)j.x + line * j.pitch + c.col, n);
        else x.template load<NT>((const T*)j.x + line * j.pitch + c.from);
        if constexpr (!std::is_void<M>::value) {
            if constexpr (SHORT) m.load_short((const M*)j.mask + line * j.mask_pitch + c.col, n);
            else m.template load<NT>((const M*)j.mask + line * j.mask_pitch + c.from);
        }
    }
    __device__ __forceinline__ void settle(const Columns& c)
    {
        if (SHORT || c.down == 0) return;
        x.down(c.down);
        if constexpr (!std::is_void<M>::value) m.down(c.down);
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (!std::is_void<M>::value) return m[i] > 0.f ? x[i] : 0.f;
        else return x[i];
    }
};

// Which 64 columns a block takes, and which of `parts` pieces of the contraction: neighbouring columns of a piece follow one another on one
// XCD, whose L2 then has the lines that two blocks share.  (Pieces of the same columns in turn, us a backward pass: 12305 tokens 523 -> 1195
// 104.0 against 94.9, 6376 tokens 2189 -> 3610 247.9 against 224.3; 8192 tokens 4096 -> 4096, no line shared, 351 against 346.)
__device__ __forceinline__ unsigned column_tile(const Job& j, unsigned block, unsigned parts, unsigned* piece)
{
    const unsigned tiles = (unsigned)((j.rows + 63) / 64), at = (unsigned)xcd_band((int)block, (int)(tiles * parts));
    *piece = at / tiles;
    return at - *piece * tiles;
}

// First launch: a block leaves the largest value and the sum of 64 columns over one part of the contraction.
template <class T, class M, bool SHORT> __device__ __forceinline__ void parts_loop(const Job& j, const Columns& col, int64_t from, int64_t to, int group,
                                                                       unsigned (&top)[across<T>()], double (&total)[across<T>()])
{
    constexpr int V = across<T>(), STEP = groups<T>(), AHEAD = SHORT ? 1 : std::is_void<M>::value ? 8 : 4;
    for (int64_t piece = from + group; piece < to; piece += 64 * STEP) {     // float32 sums of 64 values, added in float64
        float s[V] = {};
        const int64_t end = piece + 64 * STEP < to ? piece + 64 * STEP : to;
        int64_t k = piece;
        auto see = [&](const Masked<T, M, SHORT, false>& v) {
#pragma unroll
            for (int e = 0; e < V; ++e) { const float f = v[e]; top[e] = max(top[e], abs_bits(f)); s[e] += f; }
        };
        for (; k + (AHEAD - 1) * STEP < end; k += AHEAD * STEP) {
            Masked<T, M, SHORT, false> v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v[i].load(j, k + i * STEP, col);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) { v[i].settle(col); see(v[i]); }
        }
        for (; k < end; k += STEP) {
            Masked<T, M, SHORT, false> v;
            v.load(j, k, col);
            v.settle(col);
            see(v);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) total[e] += s[e];
    }
}
template <class T, bool SHORT> __device__ __forceinline__ void parts_role(const Job& j, unsigned block, Shared& sh)
{
    constexpr int V = across<T>(), LANES = 64 / V, GROUPS = groups<T>();
    unsigned part;
    const unsigned tile = column_tile(j, block, (unsigned)j.parts, &part);
    const int c = (threadIdx.x % LANES) * V, group = threadIdx.x / LANES;
    const int64_t col = (int64_t)tile * 64 + c;
    const int64_t from = part * j.per_part, to = from + j.per_part < j.len ? from + j.per_part : j.len;
    unsigned top[V] = {};
    double total[V] = {};
    if (col < j.rows) {
        const Columns mine = columns_of<T>(col, j.rows);
        if (!j.mask) parts_loop<T, void, SHORT>(j, mine, from, to, group, top, total);
        else if (j.mask_bf16) parts_loop<T, bf16, SHORT>(j, mine, from, to, group, top, total);
        else parts_loop<T, float, SHORT>(j, mine, from, to, group, top, total);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) { sh.parts.tops[group][c + i] = top[i]; sh.parts.sums[group][c + i] = (float)total[i]; }
    __syncthreads();
    const int64_t mine = (int64_t)tile * 64 + threadIdx.x;
    if (threadIdx.x < 64 && mine < j.rows) {
        unsigned t = 0;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) { t = max(t, sh.parts.tops[i][threadIdx.x]); s += sh.parts.sums[i][threadIdx.x]; }
        if (j.part_max) j.part_max[(int64_t)part * j.rows + mine] = __uint_as_float(t);
        if (j.part_sum) j.part_sum[(int64_t)part * j.rows + mine] = (float)s;
    }
}

// Second launch: tiles of 64 columns x 128 positions, several of them one after the other where there are many, the next one's loads under
// way while one is stored.  A thread takes POS neighbouring positions of its columns: words of four codes for each of them.
template <class T, class M, bool SHORT> __device__ __forceinline__ void turn_tiles(const Job& j, int64_t row0, unsigned len_tile, unsigned count, Shared& sh)
{
    constexpr int V = across<T>(), LANES = 64 / V, POS = 128 / groups<T>();
    const int c = (threadIdx.x % LANES) * V, group = threadIdx.x / LANES;
    const Columns col = columns_of<T>(row0 + c, j.rows);
    Masked<T, M, SHORT, true> v[POS];
    auto load = [&](unsigned tile) {       // (positions behind the last one: the last one, and codes of 0 below)
        const int64_t k = (int64_t)tile * 128 + group * POS;
#pragma unroll
        for (int i = 0; i < POS; ++i) v[i].load(j, k + i < j.len ? k + i : j.len - 1, col);
    };
    load(len_tile);
    // the parts' largest values, and the multipliers
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t mine = row0 + lane;
    unsigned top = 0;
    if (mine < j.rows)
#pragma unroll 8
        for (int p = wave; p < j.parts; p += 4) top = max(top, __float_as_uint(j.part_max[(int64_t)p * j.rows + mine]));
    sh.turn.tops[wave][lane] = top;
    __syncthreads();
    if (wave == 0) {
        float s;
        sh.turn.mult[lane] = row_multiplier(max(max(sh.turn.tops[0][lane], sh.turn.tops[1][lane]), max(sh.turn.tops[2][lane], sh.turn.tops[3][lane])), &s);
        if (len_tile == 0 && mine < j.rows) j.scale[mine] = s;
    }
    __syncthreads();
    float mult[V];
#pragma unroll
    for (int i = 0; i < V; ++i) mult[i] = sh.turn.mult[c + i];
    for (unsigned t = 0; t < count; ++t) {
        unsigned (&tile)[64][33] = sh.turn.tile[t & 1];
#pragma unroll
        for (int i = 0; i < POS; ++i) v[i].settle(col);
        const int64_t k = (int64_t)(len_tile + t) * 128 + group * POS;
        const int left = j.len - k < POS ? (j.len > k ? (int)(j.len - k) : 0) : POS;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int h = 0; h < POS / 4; ++h) {
                unsigned w = pack4(code_of(v[h * 4][i], mult[i]), code_of(v[h * 4 + 1][i], mult[i]), code_of(v[h * 4 + 2][i], mult[i]),
                                   code_of(v[h * 4 + 3][i], mult[i]));
                if (left < POS) w = left <= h * 4 ? 0u : left >= h * 4 + 4 ? w : w & (0xffffffffu >> (8 * (h * 4 + 4 - left)));
                tile[c + i][group * (POS / 4) + h] = w;
            }
        if (t + 1 < count) load(len_tile + t + 1);
        __syncthreads();          // (one a tile is enough: the tile after next is written behind the next one's)
#pragma unroll
        for (int h = 0; h < 2; ++h) {           // a row's 128 bytes by eight lanes
            const int u = threadIdx.x + h * 256, rr = u >> 3, w = (u & 7) * 4;
            const int64_t row = row0 + rr, at = (int64_t)(len_tile + t) * 128 + w * 4;
            if (row < j.rows && at < j.q_pitch)
                *(uint4*)(j.q + row * j.q_pitch + at) = make_uint4(tile[rr][w], tile[rr][w + 1], tile[rr][w + 2], tile[rr][w + 3]);
        }
    }
}
template <class T, bool SHORT> __device__ __forceinline__ void turn_role(const Job& j, unsigned block, Shared& sh)
{
    unsigned len_block;
    const unsigned row_tile = column_tile(j, block, j.len_blocks, &len_block), first = len_block * j.tiles_each;
    const unsigned count = min(j.tiles_each, j.len_tiles - first);
    const int64_t row0 = (int64_t)row_tile * 64;
    if (j.sum && first == 0) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        double total = 0.0;
        if (row0 + lane < j.rows)
            for (int p = wave; p < j.parts; p += 4) total += j.part_sum[(int64_t)p * j.rows + row0 + lane];
        sh.turn.sums[wave][lane] = total;
        __syncthreads();
        if (wave == 1 && row0 + lane < j.rows)
            j.sum[row0 + lane] = (float)((sh.turn.sums[0][lane] + sh.turn.sums[1][lane]) + (sh.turn.sums[2][lane] + sh.turn.sums[3][lane]));
    }
    if (!j.q) return;
    if (!j.mask) turn_tiles<T, void, SHORT>(j, row0, first, count, sh);
    else if (j.mask_bf16) turn_tiles<T, bf16, SHORT>(j, row0, first, count, sh);
    else turn_tiles<T, float, SHORT>(j, row0, first, count, sh);
}

template <class T> __device__ __forceinline__ void rows_any(const Job& j, unsigned block, Shared& sh)
{
    const int lanes = row_lanes(j.len, sizeof(T) == 2);
    if (lanes == 32) rows_role<T, 32, 4>(j, block, sh);
    else if (lanes == 64) rows_role<T, 64, row_keep<T>()>(j, block, sh);
    else rows_role<T, 256, 4>(j, block, sh);
}
template <class T> __device__ __forceinline__ void first_role(const Job& j, unsigned block, Shared& sh)
{
    if (!j.along) { if (j.rows < across<T>()) parts_role<T, true>(j, block, sh); else parts_role<T, false>(j, block, sh); }
    else rows_any<T>(j, block, sh);
}
__global__ __launch_bounds__(256, 3) void k_quantize_first(const Jobs jobs)
{
    __shared__ Shared sh;
    int i = 0;
    while (i + 1 < jobs.n && blockIdx.x >= jobs.first1[i + 1]) ++i;
    const Job& j = jobs.job[i];
    if (j.bf16_) first_role<bf16>(j, blockIdx.x - jobs.first1[i], sh); else first_role<float>(j, blockIdx.x - jobs.first1[i], sh);
}
// one source that lies along memory: the forward pass
template <class T, int LANES, int KEEP> __global__ __launch_bounds__(256) void k_quantize_rows(const Job j)
{
    __shared__ Shared sh;
    rows_role<T, LANES, KEEP, true>(j, blockIdx.x, sh);
}
template <class T> static void rows_launch(Ctx& c, const Job& j, unsigned blocks)
{
    switch (row_lanes(j.len, sizeof(T) == 2)) {
    case 32: ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, 32, 4>), dim3(blocks), dim3(256), 0, j); break;
    case 64: ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, 64, row_keep<T>()>), dim3(blocks), dim3(256), 0, j); break;
    default: ST_LAUNCH(c, "quantize_rows", (k_quantize_rows<T, 256, 4>), dim3(blocks), dim3(256), 0, j);
    }
}
__global__ __launch_bounds__(256, 4) void k_quantize_turn(const Jobs jobs)
{
    __shared__ Shared sh;
    int i = 0;
    while (i + 1 < jobs.n && blockIdx.x >= jobs.first2[i + 1]) ++i;
    const Job& j = jobs.job[i];
    const unsigned block = blockIdx.x - jobs.first2[i];
    if (j.bf16_) { if (j.rows < across<bf16>()) turn_role<bf16, true>(j, block, sh); else turn_role<bf16, false>(j, block, sh); }
    else         { if (j.rows < across<float>()) turn_role<float, true>(j, block, sh); else turn_role<float, false>(j, block, sh); }
}

// ------------------------------------------------------------------------------------------------------------- host
// Two blocks a compute unit, parts of 64 positions at least: the second launch reads every part's value of each of its rows.  (Four, us a
// call: 11244 tokens 1402 -> 131 that lie across memory 37.4 against 34.4; two of three backward passes gain up to 5 %, the others lose up to 4.)
int transpose_parts(int64_t rows, int64_t len)
{
    const int64_t across = ceil_div(rows, 64), most = ceil_div(len, 64);
    int64_t parts = ceil_div(512, across);
    if (parts > 128) parts = 128;
    return (int)(parts > most ? most : parts < 1 ? 1 : parts);
}

void quantize(Ctx& c, const QuantTask* tasks, int n)
{
    Jobs jobs;
    jobs.n = 0;
    // sources that lie along memory first, so that the second launch has the others in consecutive places
    int64_t blocks1 = 0, blocks2 = 0;
    for (int pass = 1; pass >= 0; --pass)
        for (int i = 0; i < n; ++i) {
            const QuantTask& t = tasks[i];
            const QuantSource& s = t.s;
            if (s.along != pass || s.rows == 0) continue;
            jobs.first1[jobs.n] = (unsigned)blocks1; jobs.first2[jobs.n] = (unsigned)blocks2;
            Job& j = jobs.job[jobs.n++];
            j = Job{s.x, s.mask, s.pitch, s.mask_pitch, s.rows, s.len, t.to.pitch, 0, t.to.q, t.to.scale, t.sum, t.to.q ? t.part_max : nullptr,
                    t.sum ? t.part_sum : nullptr, 1, 1, 1, 1, (uint8_t)s.bf16, (uint8_t)s.mask_bf16, (uint8_t)s.along};
            if (s.along) { blocks1 += ceil_div(s.rows, 256 / row_lanes(s.len, s.bf16)); continue; }
            j.parts = transpose_parts(s.rows, s.len);
            j.per_part = ceil_div(s.len, j.parts);
            j.len_tiles = t.to.q ? (unsigned)ceil_div(s.len, 128) : 1;
            j.tiles_each = (unsigned)std::min<int64_t>(4, std::max<int64_t>(1, ceil_div(s.rows, 64) * j.len_tiles / 1024));
            j.len_blocks = (unsigned)ceil_div(j.len_tiles, j.tiles_each);
            blocks1 += ceil_div(s.rows, 64) * j.parts;
            blocks2 += ceil_div(s.rows, 64) * j.len_blocks;
        }
    if (jobs.n == 1 && jobs.job[0].along) {
        if (jobs.job[0].bf16_) rows_launch<bf16>(c, jobs.job[0], (unsigned)blocks1); else rows_launch<float>(c, jobs.job[0], (unsigned)blocks1);
    } else if (blocks1) ST_LAUNCH(c, "quantize_first", k_quantize_first, dim3((unsigned)blocks1), dim3(256), 0, jobs);
    if (!blocks2) return;
    Jobs turn;
    turn.n = 0;
    for (int i = 0; i < jobs.n; ++i)
        if (!jobs.job[i].along) { turn.first2[turn.n] = jobs.first2[i]; turn.job[turn.n++] = jobs.job[i]; }
    ST_LAUNCH(c, "quantize_turn", k_quantize_turn, dim3((unsigned)blocks2), dim3(256), 0, turn);
}

__global__ __launch_bounds__(256) void k_fill_zero(float* __restrict__ p, int64_t rows, int64_t cols, int64_t pitch)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256) p[i / cols * pitch + i % cols] = 0.f;
}
void fill_zero(Ctx& c, float* p, int64_t rows, int64_t cols, int64_t pitch)
{
    const int64_t blocks = ceil_div(rows * cols, 2048);
    ST_LAUNCH(c, "fill_zero", k_fill_zero, dim3((unsigned)(blocks > 4096 ? 4096 : blocks)), dim3(256), 0, p, rows, cols, pitch);
}

}  // namespace st
